"""A small server of prompts of different lengths over the paged 8-bit KV cache.

One attention stack (QKV projection, attention, output projection and residual per layer) serves a batch of prompts the
way a block-diffusion or single-token decoder does:

1. the prompts are packed, attended causally (``tadm_attention_packed``) and stored in pages (``tadm_page_write``);
2. every prompt is forked into branches that share its full pages (``tadm_pages_fork``);
3. each branch appends blocks of tokens: pages are reserved, the block's keys and values stored, and its rows attend over
   the cache, bidirectionally within the block (``tadm_page_attention``);
4. all branches but the first of each prompt are freed and the pool is compacted (``tadm_pages_free``,
   ``tadm_pages_compact``); the survivors go on, one token at a time.

    python examples/ragged_server.py [--layers 4] [--prompts 6] [--branches 3] [--block 32] [--blocks 2]

``--check`` recomputes every layer's attention in 64 bits from the rows that were stored (through ``tadm_page_read``)
and prints the largest relative error.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2609_37924_gb300 import tadm as T  # noqa: E402

PAGE = T.PAGE_TOKENS


class Server:
    """Layers of attention over one page pool; sequences are rows of one page table."""

    def __init__(self, layers=4, heads=16, kv_heads=8, hd=128, seqs=24, max_len=2048, pages=256, seed=0, check=False):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        d = heads * hd
        rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.wqkv = [(rand((heads + 2 * kv_heads) * hd, d) / math.sqrt(d)).bfloat16() for _ in range(layers)]
        self.wo = [(rand(d, d) / math.sqrt(d)).bfloat16() for _ in range(layers)]
        self.heads, self.kv_heads, self.hd, self.layers, self.max_len = heads, kv_heads, hd, layers, max_len
        self.pool = T.PagePool.empty(layers, pages, kv_heads, hd)
        self.tables = torch.full((seqs, max_len // PAGE), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.scratch = torch.empty(T.tadm_pages_scratch_size(pages, seqs), dtype=torch.uint8, device="cuda")
        self.check, self.worst = check, 0.0

    def ints(self, values):
        return torch.tensor(list(values), dtype=torch.int32, device="cuda")

    def done(self, what):
        if int(self.status) != 0:
            raise RuntimeError(f"{what}: status {int(self.status)} (1: no free pages, 2: inconsistent request)")

    # -- bookkeeping, all of it in place ---------------------------------------------------------
    def reserve(self, seqs, new_len):
        T.tadm_pages_reserve(self.tables, self.refs, self.ints(seqs), self.ints(new_len), self.tables, self.refs,
                             self.status, self.scratch)
        self.done("reserve")

    def fork(self, src, dst):
        T.tadm_pages_fork(self.pool, self.tables, self.lens, self.refs, self.ints(src), self.ints(dst), self.tables,
                          self.lens, self.refs, self.status, self.scratch)
        self.done("fork")

    def free(self, seqs):
        T.tadm_pages_free(self.tables, self.lens, self.refs, self.ints(seqs), self.tables, self.lens, self.refs,
                          self.status, self.scratch)
        self.done("free")

    def compact(self) -> int:
        T.tadm_pages_compact(self.pool, self.tables, self.refs, self.tables, self.refs, self.status, self.scratch)
        return int(self.status)

    # -- layers ----------------------------------------------------------------------------------
    def project(self, x, layer):
        qkv = torch.empty((x.shape[0], self.wqkv[layer].shape[0]), dtype=torch.bfloat16, device="cuda")
        n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        T.tadm_gemm(n.bfloat16(), self.wqkv[layer], qkv, dtype=1)
        qkv = qkv.view(x.shape[0], self.heads + 2 * self.kv_heads, self.hd)
        return qkv[:, :self.heads], qkv[:, self.heads:self.heads + self.kv_heads], qkv[:, self.heads + self.kv_heads:]

    def output(self, x, o, layer):
        y = torch.empty_like(x)
        T.tadm_gemm(o.view(x.shape[0], -1), self.wo[layer], y, dtype=1)
        return x + y

    def prefill(self, x, seqs, lens):
        """Whole prompts, packed: x fp32 [sum(lens), d]; they become tokens 0 .. of the (empty) sequences seqs."""
        self.reserve(seqs, lens)
        cu, start = self.ints(_cum(lens)), self.ints([0] * len(lens))
        table = self.tables[self.ints(seqs).long()].contiguous()
        for layer in range(self.layers):
            q, k, v = self.project(x, layer)
            o = torch.empty((x.shape[0], self.heads, self.hd), dtype=torch.bfloat16, device="cuda")
            T.tadm_attention_packed(q, k, v, o, cu, max(lens))
            T.tadm_page_write(self.pool, layer, k, v, cu, start, table, max(lens))
            x = self.output(x, o, layer)
        self.lens[self.ints(seqs).long()] = self.ints(lens)
        return x

    def step(self, x, seqs, rows, causal=False):
        """`rows` new tokens of every sequence of seqs: x fp32 [len(seqs) * rows, d]."""
        at = self.ints(seqs).long()
        old = self.lens[at].tolist()
        new = [n + rows for n in old]
        self.reserve(seqs, new)
        table, cu = self.tables[at].contiguous(), self.ints(_cum([rows] * len(seqs)))
        start, lens = self.ints(old), self.ints(new)
        need = T.tadm_page_attention_scratch_size(len(seqs), x.shape[0], rows, max(new), self.heads, self.kv_heads, self.hd, 1)
        scratch = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        for layer in range(self.layers):
            q, k, v = self.project(x, layer)
            o = torch.empty((x.shape[0], self.heads, self.hd), dtype=torch.bfloat16, device="cuda")
            T.tadm_page_write(self.pool, layer, k, v, cu, start, table, rows)
            T.tadm_page_attention(q, self.pool, layer, o, cu, lens, table, rows, max(new), scratch, causal=causal)
            if self.check:
                self.compare(q, o, layer, table, new, rows, causal)
            x = self.output(x, o, layer)
        self.lens[at] = lens
        return x

    def compare(self, q, o, layer, table, lens, rows, causal):
        k = torch.empty((sum(lens), self.kv_heads, self.hd), dtype=torch.bfloat16, device="cuda")
        v = torch.empty_like(k)
        T.tadm_page_read(self.pool, layer, k, v, self.ints(_cum(lens)), self.ints([0] * len(lens)), table, max(lens))
        for b, n in enumerate(lens):
            at = _cum(lens)[b]
            kk, vv = (t[at:at + n].double().repeat_interleave(self.heads // self.kv_heads, 1) for t in (k, v))
            s = torch.einsum("rhd,nhd->hrn", q[b * rows:(b + 1) * rows].double(), kk) / math.sqrt(self.hd)
            if causal:
                pos = torch.arange(n - rows, n, device="cuda")[:, None]
                s = s.masked_fill(torch.arange(n, device="cuda") > pos, -math.inf)
            ref = torch.einsum("hrn,nhd->rhd", torch.softmax(s, -1), vv)
            got = o[b * rows:(b + 1) * rows].double()
            self.worst = max(self.worst, float((got - ref).norm() / ref.norm()))


def _cum(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def serve(layers=4, prompts=6, branches=3, block=32, blocks=2, tokens=4, heads=16, kv_heads=8, hd=128, seed=0, check=False):
    """The loop above; returns (final rows, pages in use at the peak, after the compaction, worst relative error)."""
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(1, 600, (prompts,), generator=g).tolist()
    s = Server(layers, heads, kv_heads, hd, seqs=prompts * branches, max_len=1024, pages=prompts * branches * 16, seed=seed, check=check)
    rand = lambda n: torch.randn((n, heads * hd), generator=g).cuda()  # noqa: E731
    first = list(range(prompts))
    s.prefill(rand(sum(lens)), first, lens)
    others = list(range(prompts, prompts * branches))
    s.fork([i % prompts for i in others], others)
    every = first + others
    for _ in range(blocks):
        x = s.step(rand(len(every) * block), every, block)
    peak = int((s.refs > 0).sum())
    s.free(others)
    live = s.compact()
    for _ in range(tokens):
        x = s.step(rand(len(first)), first, 1, causal=True)
    T.tadm_ragged_sync_status()
    assert s.lens.tolist() == [n + blocks * block + tokens for n in lens] + [0] * len(others)
    return x, peak, live, s.worst


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("prompts", 6), ("branches", 3), ("block", 32), ("blocks", 2), ("tokens", 4), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    import __graft_entry__ as g
    g.build()
    x, peak, live, worst = serve(a.layers, a.prompts, a.branches, a.block, a.blocks, a.tokens, seed=a.seed, check=a.check)
    torch.cuda.synchronize()
    print(f"{a.prompts} prompts x {a.branches} branches, {a.blocks} blocks of {a.block}, then {a.tokens} tokens: "
          f"{peak} pages at the peak, {live} after the compaction, finite: {bool(torch.isfinite(x).all())}"
          + (f", attention within {worst:.1e} of 64 bits" if a.check else ""))


if __name__ == "__main__":
    main()
