"""Eviction's bookkeeping on host-only caches, against a list model: pages popped before the old ones go back, sinks'
pages kept, reference counts under forks, checkpoints, failures undone; and what is refused.  An 8-bit cache keeps
the same books as a bf16 one."""
import random

import pytest

import paper_2609_04875_gb300 as pe


class Books:
    """Free list (top last), tables, lengths, references, by the rules of pe_evict_batch."""

    def __init__(self, ps, pages, seqs, max_pages, bits):
        self.ps = ps
        self.cache = pe.PagedKVCache(2, 2, 64, ps, pages, seqs, max_pages, host_only=True, kv_bits=bits)
        self.free = list(range(pages))[::-1]
        self.table, self.len, self.refs = {}, {}, [0] * pages

    def append(self, s, n):
        self.cache.append_kv(s, n_tokens=n)
        t = self.table[s]
        if n and self.len[s] % self.ps and self.refs[t[-1]] > 1:
            self.refs[t[-1]] -= 1
            t[-1] = self.free.pop()
            self.refs[t[-1]] = 1
        self.len[s] += n
        while len(t) < -(-self.len[s] // self.ps):
            t.append(self.free.pop())
            self.refs[t[-1]] = 1

    def new(self):
        s = self.cache.seq_create()
        self.table[s], self.len[s] = [], 0
        return s

    def fork(self, s):
        f = self.cache.seq_fork(s)
        self.table[f], self.len[f] = list(self.table[s]), self.len[s]
        for p in self.table[s]:
            self.refs[p] += 1
        return f

    def evict(self, seqs, keep, sinks, recent, done=False):
        if not done:
            self.cache.evict_batch(seqs, keep, sinks=sinks, recent=recent)
        fresh = {}
        for s, k in zip(seqs, keep):
            if k < self.len[s]:
                fresh[s] = [self.free.pop() for _ in range(-(-k // self.ps) - sinks // self.ps)]
        for s, k in zip(seqs, keep):
            if s in fresh:
                first = sinks // self.ps
                for p in self.table[s][first:][::-1]:
                    self.refs[p] -= 1
                    if self.refs[p] == 0:
                        self.free.append(p)
                for p in fresh[s]:
                    self.refs[p] = 1
                self.table[s] = self.table[s][:first] + fresh[s]
                self.len[s] = k

    def check(self):
        assert self.cache.free_list() == self.free[::-1]
        assert self.cache.page_refs() == self.refs
        for s, t in self.table.items():
            assert self.cache.page_table(s) == t
            assert self.cache.seq_info(s)[0] == self.len[s]


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("ps", [8, 16, 128])
def test_random_evictions(ps, bits):
    r = random.Random(ps)
    b = Books(ps, 400, 12, 60, bits)
    seqs = [b.new() for _ in range(3)]
    for step in range(150):
        what = r.random()
        s = r.choice(seqs)
        if what < 0.4:
            n = r.randrange(0, 6 * ps)
            if len(b.free) > 8 and b.len[s] + n <= 50 * ps:
                b.append(s, n)
        elif what < 0.55 and len(seqs) < 12:
            seqs.append(b.fork(s))
        else:
            batch = r.sample(seqs, r.randrange(1, min(4, len(seqs)) + 1))
            sinks, recent = r.choice([0, 1, ps, 2 * ps + 1]), r.choice([0, 3, ps])
            keep = [max(sinks + recent, r.randrange(0, b.len[q] + 2)) for q in batch]
            need = sum(-(-k // ps) - sinks // ps for k, q in zip(keep, batch) if k < b.len[q])
            before = b.cache.free_list()
            if need > len(b.free):
                with pytest.raises(pe.PEError) as e:
                    b.cache.evict_batch(batch, keep, sinks=sinks, recent=recent)
                assert e.value.kind == "oom" and b.cache.free_list() == before
                continue
            done = False
            if r.random() < 0.3:  # a device step fails: nothing changed
                b.cache.set_option("fail_launch_after", r.randrange(3))
                try:
                    b.cache.evict_batch(batch, keep, sinks=sinks, recent=recent)
                    done = True  # the call had fewer steps than that
                except pe.PEError as e:
                    assert e.kind == "cuda"
                    b.check()
                b.cache.set_option("fail_launch_after", -1)
            b.evict(batch, keep, sinks, recent, done)
        b.check()


def test_checkpoints_past_the_sinks_go():
    b = Books(16, 40, 2, 20, 8)
    s = b.new()
    b.append(s, 100)
    for o in (0, 5, 10, 11, 50, 100):
        b.cache.checkpoint_add(s, o)
    b.cache.evict_batch([s], [60], sinks=10, recent=5)
    assert b.cache.checkpoints(s) == [0, 5, 10]
    assert b.cache.seq_info(s) == (60, 100)
    b.cache.evict_batch([s], [60], sinks=0)       # it has no more than that: nothing changes
    assert b.cache.checkpoints(s) == [0, 5, 10]


def test_refusals():
    b = Books(16, 12, 2, 12, 8)
    s, t = b.new(), b.new()
    b.append(s, 100)
    b.append(t, 20)
    for kind, seqs, keep, kw in [("invalid", [s, s], [5, 5], {}), ("invalid", [3], [5], {}), ("invalid", [s], [-1], {}),
                                 ("invalid", [s], [5], {"sinks": 3, "recent": 3}), ("invalid", [s], [5], {"recent": -1}),
                                 ("oom", [s], [90], {})]:
        with pytest.raises(pe.PEError) as e:
            b.cache.evict_batch(seqs, keep, **kw)
        assert e.value.kind == kind
        b.check()
    with pytest.raises(ValueError):
        b.cache.read_kv(s)
    with pytest.raises(ValueError):
        pe.PagedKVCache(1, 1, 64, 16, 4, 1, 4, host_only=True, kv_bits=12)
    b.cache.evict_batch([], [])
