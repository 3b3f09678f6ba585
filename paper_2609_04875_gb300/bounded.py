"""Agents with bounded sessions: K and V in 8 bits, an account of every key's softmax weight, and eviction when a session
passes its budget.  A forget request names a position of the whole session: the driver keeps each held token's.

    python -m paper_2609_04875_gb300.bounded        # a short synthetic run, one GPU

One step of every agent is: append its token to all layers, attend it layer by layer (each call adds the keys' weights
to the agent's account), and, once a session is longer than ``budget + slack``, come down to ``budget`` tokens: the
first ``sinks``, the last ``recent`` and the ones that drew the most weight.  So the cache of an agent never holds more
than ``budget + slack + 1`` tokens, whatever its session's length.

A forget request leaves no held token, no later position and nothing in the account of the forgotten turns, so what is
evicted from then on does not depend on them.  Two traces stay.  Tokens that were evicted while the forgotten turns were
there, for want of the weight that those drew to others, do not come back.  And kept tokens that share the last page with
forgotten ones stay rounded to a scale that those may have set; a request on a page's end has no such tokens.
"""
from __future__ import annotations

import torch

from .binding import PagedKVCache, Rope


class BoundedAgents:
    def __init__(self, agents, layers, hq, hkv, d, budget, slack=256, sinks=4, recent=64, page_size=16, longest_prompt=None,
                 rope=None):
        """``rope`` (binding.Rope): K and Q come unrotated, and turn by each token's position in its whole session (on every
        axis), which eviction does not change."""
        if sinks + recent > budget:
            raise ValueError("sinks + recent exceed the budget")
        self.layers, self.hq, self.budget, self.slack, self.sinks, self.recent = layers, hq, budget, slack, sinks, recent
        self.columns = max(budget + slack + 1, longest_prompt or 0)
        pages = -(-self.columns // page_size) + 1
        # an eviction copies into fresh pages before it frees the old ones: a budget's worth for every agent
        self.cache = PagedKVCache(layers, hkv, d, page_size, agents * (pages + -(-budget // page_size) + 1), agents, pages,
                                  kv_bits=8)
        self.seqs = [self.cache.seq_create() for _ in range(agents)]
        self.weights = torch.zeros((agents, self.columns), device="cuda")
        # origin[i][j]: the position in agent i's whole session of the token its cache holds at position j
        self.origin = torch.full((agents, self.columns), -1, dtype=torch.int32, device="cuda")
        self.seen = [0] * agents
        self.rope = rope

    def lengths(self):
        return [self.cache.seq_info(s)[0] for s in self.seqs]

    def append(self, K, V, Q, counts):
        """counts[i] tokens of each agent: K, V bf16 [L][sum][Hkv][d], Q bf16 [L][sum][Hq][d], packed agent by agent.
        Returns the attention outputs [L][sum][Hq][d] (before any eviction)."""
        cu = [0]
        for n in counts:
            cu.append(cu[-1] + n)
        lens = self.lengths()
        if max(a + n for a, n in zip(lens, counts)) > self.columns:
            raise ValueError("more tokens than a session may hold at once")
        # where the new tokens are held, and their positions in the whole sessions
        new = [(i, a + j, seen + j) for i, (a, n, seen) in enumerate(zip(lens, counts, self.seen)) for j in range(n)]
        rows, at, pos = torch.tensor(new, dtype=torch.int64, device="cuda").reshape(-1, 3).t()
        pos = pos.int()
        if self.rope is None:
            self.cache.append_kv_batch(self.seqs, K, V, cu)
        else:
            Q = self.cache.append_kv_rope_batch(self.seqs, K, V, cu, self.rope, Q=Q, positions=self._on_axes(pos))
        if new:
            self.origin[rows, at] = pos
        self.seen = [a + n for a, n in zip(self.seen, counts)]
        out = torch.empty_like(Q)
        for layer in range(self.layers):
            self.cache.replay_attn_weights_batch(self.seqs, layer, Q[layer], cu, self.weights, out=out[layer])
        self._evict()
        return out

    def _on_axes(self, pos):
        return pos.expand(self.rope.n_axes, -1).contiguous()

    def _evict(self):
        over = [i for i, n in enumerate(self.lengths()) if n > self.budget + self.slack]
        if not over:
            return
        rows = torch.tensor(over, device="cuda")
        w, keep = self.weights[rows], [self.budget] * len(over)
        kept = self.cache.evict_batch([self.seqs[i] for i in over], keep, w, sinks=self.sinks, recent=self.recent)
        self.weights[rows] = w
        moved = torch.full_like(w, -1, dtype=torch.int32)
        moved[:, : self.budget] = torch.gather(self.origin[rows], 1, kept.long())
        self.origin[rows] = moved

    def forget(self, agent, tau):
        """Crops the agent to the held tokens that stood before position tau (1-based) of its whole session; returns how
        many those are.  Their K and V may be replayed from there.  The account starts anew, since the forgotten turns'
        queries are in every key's sum (recount fills it from the kept ones)."""
        if not 1 <= tau <= self.seen[agent] + 1:
            raise ValueError("tau outside the session")
        held = self.lengths()[agent]
        keep = int((self.origin[agent, :held] < tau - 1).sum())  # (positions ascend: eviction keeps the order)
        self.cache.crop(self.seqs[agent], keep + 1)
        self.weights[agent] = 0
        self.origin[agent, keep:] = -1
        self.seen[agent] = tau - 1
        return keep

    def recount(self, agent, Q):
        """The agent's account from its held tokens' queries alone, Q bf16 [L][held][Hq][d]."""
        held = self.lengths()[agent]
        if tuple(Q.shape) != (self.layers, held, self.hq, self.cache.head_dim):
            raise ValueError(f"Q must be [{self.layers}][{held}][{self.hq}][{self.cache.head_dim}]")
        self.weights[agent] = 0
        if self.rope is not None:
            Q = self.cache.rotate(self.seqs[agent], Q, self.rope, positions=self._on_axes(self.origin[agent, :held]))
        for layer in range(self.layers if held else 0):
            self.cache.replay_attn_weights_batch([self.seqs[agent]], layer, Q[layer], [0, held], self.weights[agent: agent + 1])


def main():
    agents, layers, hq, hkv, d = 8, 2, 32, 8, 128
    rope = Rope([10000.0 ** (-i / (d // 2)) for i in range(d // 2)])
    b = BoundedAgents(agents, layers, hq, hkv, d, budget=1024, slack=128, longest_prompt=3000, rope=rope)
    g = torch.Generator("cuda").manual_seed(1)

    def tokens(counts):
        n = sum(counts)
        draw = lambda h: torch.randn((layers, n, h, d), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
        return draw(hkv), draw(hkv), draw(hq), counts

    b.append(*tokens([3000 - 100 * i for i in range(agents)]))
    print("after the prompts:", b.lengths())
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    steps = [tokens([1] * agents) for _ in range(300)]
    torch.cuda.synchronize()
    start.record()
    for s in steps:
        b.append(*s)
    end.record()
    torch.cuda.synchronize()
    print("after 300 steps:", b.lengths(), f"{start.elapsed_time(end) / 300 * 1e3:.0f} us a step of {agents} agents x {layers} layers")
    kept = b.forget(2, 2900)
    print("agent 2 forgets from position 2900 on:", kept, "tokens held before it")
    b.recount(2, tokens([kept])[2])  # (a program has the kept tokens' queries from their replay)
    b.append(*tokens([1] * agents))
    assert b.cache.device_status() == 0


if __name__ == "__main__":
    main()
