"""pe_replay_attn_static_scratch allocates nothing, on the host either: no operator new of the process runs inside it."""
import os
import subprocess
import sys

import pytest

from gpu_common import requires_cuda

pytestmark = [pytest.mark.gpu, requires_cuda]


COUNT_NEW = """
#include <cstdlib>
#include <new>
static long count = 0;
extern "C" long operator_news() { return count; }
void *operator new(std::size_t n) { ++count; void *p = std::malloc(n ? n : 1); if (!p) std::abort(); return p; }
void *operator new[](std::size_t n) { return operator new(n); }
void operator delete(void *p) noexcept { std::free(p); }
void operator delete[](void *p) noexcept { std::free(p); }
void operator delete(void *p, std::size_t) noexcept { std::free(p); }
void operator delete[](void *p, std::size_t) noexcept { std::free(p); }
"""
STATIC_SCRATCH = """
import ctypes, sys
import torch
import paper_2609_04875_gb300 as pe
from paper_2609_04875_gb300 import binding
count = ctypes.CDLL(None).operator_news
count.restype = ctypes.c_long
for bits in (16, 8):
    c = pe.PagedKVCache(2, 2, 64, 16, 64, 2, 64, kv_bits=bits)
    s = c.seq_create()
    k = torch.randn((2, 300, 2, 64), device="cuda").to(torch.bfloat16)
    c.append_kv(s, k, k)
    q = torch.randn((20, 4, 64), device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    args = (c.handle, s, 1, ctypes.c_void_p(q.data_ptr()), ctypes.c_void_p(out.data_ptr()), 20, 4, 0.125, None)
    fn = binding.lib().pe_replay_attn_static_scratch
    assert fn(*args) == 0
    torch.cuda.synchronize()
    before = count()
    assert before > 0
    assert fn(*args) == 0
    print(bits, count() - before)
    torch.cuda.synchronize()
"""


def test_the_static_scratch_call_allocates_nothing(tmp_path):
    """No operator new runs inside the call, on either kind of cache (its first call on a device aside)."""
    src, so = tmp_path / "count_new.cpp", tmp_path / "count_new.so"
    src.write_text(COUNT_NEW)
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", str(src), "-o", str(so)], check=True)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, LD_PRELOAD=str(so), PYTHONPATH=root)
    run = subprocess.run([sys.executable, "-c", STATIC_SCRATCH], env=env, cwd=root, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
    assert run.stdout.split() == ["16", "0", "8", "0"]
