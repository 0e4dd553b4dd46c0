"""A server's loop over a packed cache: several samples of one prompt, by draft-and-verify steps.

    python examples/packed_serving.py [--samples 6] [--steps 8] [--prompt 1000]

The prompt's keys and values are appended once, in 4 bits a value.  Rows of the
page table that share its pages are forked from it, each with pages of its own
for what it will add; every step appends the rows of the last token and the
drafts, attends over the packed cache, accepts drafts, gives the log
probabilities of what it emitted, and commits.  Rows that are done give their
pages back, and at the end the pages in use move together.

The model is a stand-in: its projections and logits are seeded random numbers
of a model's shapes.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_20507_gb300 import binding as cs   # noqa: E402


class StandIn:
    """What a model would compute: rows for the cache, queries and logits."""

    def __init__(self, layers, q_heads, kv_heads, vocab, dev, seed=0):
        self.layers, self.q_heads, self.kv_heads, self.vocab, self.dev = layers, q_heads, kv_heads, vocab, dev
        self.gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.gen, device=self.dev).to(torch.bfloat16)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.gen, device=self.dev)

    def kv(self, batch, rows):
        return [(self.normal(batch, rows, self.kv_heads, 128), self.normal(batch, rows, self.kv_heads, 128))
                for _ in range(self.layers)]


class Server:
    """The cache: a packed pool a layer, one page table, the pages' counts."""

    def __init__(self, model, rows, pages, page_size, max_pages):
        self.model, self.page_size = model, page_size
        dev = model.dev
        self.pools = [cs.packed_pool(pages, model.kv_heads, page_size, dev) for _ in range(model.layers)]
        self.page_pools = [t for p in self.pools for t in (p.k_codes, p.k_scales, p.v_codes, p.v_scales)]
        self.table = torch.full((rows, max_pages), -1, dtype=torch.int32, device=dev)
        self.lens = torch.zeros((rows,), dtype=torch.int32, device=dev)
        self.counts = torch.zeros((pages,), dtype=torch.int32, device=dev)

    def rows(self, ids):
        return torch.tensor(ids, dtype=torch.int32, device=self.model.dev)

    def pool_groups(self):
        """The cache's tensors, as many at a time as a call takes."""
        m = cs.CS_MAX_PAGE_POOLS
        return [self.page_pools[i:i + m] for i in range(0, len(self.page_pools), m)]

    def fork(self, src, dst, room):
        first, *rest = self.pool_groups()
        ok = cs.cs_kv_fork(first, self.table, self.lens, self.counts, self.rows(src), self.rows(dst), self.page_size, room)
        for pools in rest:
            cs.cs_kv_fork_more(pools, self.table, self.counts, len(src))
        return ok

    def prefill(self, row, n):
        """An empty row with pages for a prompt of n tokens, and the prompt's keys and values."""
        ok = self.fork([-1], [row], n)
        self.lens[row] = n
        for pool, (k, v) in zip(self.pools, self.model.kv(1, n)):
            for i in range(0, n, 4096):     # an append takes 4096 rows a request at most
                m = min(4096, n - i)
                cs.cs_packed_kv_append(k[:, i:i + m].contiguous(), v[:, i:i + m].contiguous(), pool,
                                       self.table[row:row + 1], self.rows([i + m]))
        return ok

    def step(self, rows, n_draft, temperature, n_top):
        """One draft-and-verify step of the rows [lo, hi): their emitted tokens and these tokens' log probabilities."""
        lo, hi = rows
        m, B = self.model, hi - lo
        table, lens = self.table[lo:hi], self.lens[lo:hi]
        # the drafter proposes
        draft = m.normal(B, n_draft, m.vocab)
        tokens = torch.stack([cs.cs_sample(draft[:, i].contiguous(), m.uniform(B), temperature)
                              for i in range(n_draft)], 1)
        # the target model's layers over the last token and the drafts
        lens += n_draft + 1
        for pool, (k, v) in zip(self.pools, m.kv(B, n_draft + 1)):
            cs.cs_packed_kv_append(k, v, pool, table, lens)
            q = m.normal(B, n_draft + 1, m.q_heads, 128)
            self.attended = (q, pool, cs.cs_packed_verify_attention(q, pool, table, lens, n_draft))
        target = (torch.cat((draft, m.normal(B, 1, m.vocab)), 1) + 0.5 * m.normal(B, n_draft + 1, m.vocab)).contiguous()
        out, n = cs.cs_spec_accept(target, draft, tokens, m.uniform(B, n_draft + 1), temperature)
        scores = cs.cs_logprobs(target.view(-1, m.vocab), out.view(-1), temperature, n_top)
        cs.cs_kv_commit(lens, n, n_draft)
        self.logits = target
        return out, n, scores

    def release(self, ids):
        cs.cs_kv_release(self.table, self.lens, self.counts, self.rows(ids), self.rows([0] * len(ids)), self.page_size)

    def compact(self):
        first, *rest = self.pool_groups()
        live = cs.cs_kv_compact(first, self.table, self.counts)
        for pools in rest:
            cs.cs_kv_compact_more(pools, self.table, self.counts)
        return live


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--samples", type=int, default=6)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1000)
    a = ap.parse_args(argv)
    k, ps, temperature = 4, 16, 0.8
    room = (a.steps + 1) * (k + 1)
    max_pages = (a.prompt + room) // ps + 2
    server = Server(StandIn(2, 32, 8, 32000, torch.device("cuda:0")), 1 + a.samples,
                    max_pages + a.samples * (room // ps + 2), ps, max_pages)
    with torch.no_grad():
        server.prefill(0, a.prompt)
        forked = server.fork([0] * a.samples, range(1, 1 + a.samples), room)
        assert forked.all()
        print(f"prompt of {a.prompt} tokens, {a.samples} samples: {int((server.counts > 0).sum())} pages in use")
        total = count = torch.zeros((a.samples,), device="cuda:0")
        for _ in range(a.steps):
            out, n, (lp, entropy, top, top_lp) = server.step((1, 1 + a.samples), k, temperature, 3)
            emitted = out >= 0
            total = total + lp.view_as(out).masked_fill(~emitted, 0).sum(1)
            count = count + emitted.sum(1)
        best = int((total / count).argmax())
        print(f"samples of {(server.lens[1:] - a.prompt).tolist()} committed tokens, log probabilities a token "
              f"{[round(x, 2) for x in (total / count).tolist()]}")
        server.release([r for r in range(1 + a.samples) if r != 1 + best])
        live = server.compact()
        print(f"sample {best} kept: {int(live)} pages in use, the pages from {int(live)} on free")
    return server, best


if __name__ == "__main__":
    main()
