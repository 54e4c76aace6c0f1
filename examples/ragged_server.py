"""A small server of prompts of different lengths over the paged 8-bit KV cache.

One attention stack (norm, QKV projection, attention, output projection and residual per layer) serves a batch of prompts
the way a block-diffusion or single-token decoder does.  Every prompt has a low-rank adapter of its own or none: the
projections are ``tadm_lora_project``, and ``tadm_residual_norm`` adds a layer's output and normalises for the next:

1. the prompts are packed, attended causally (``tadm_attention_packed``) and stored in pages (``tadm_page_write``);
2. every prompt is forked into branches that share its full pages (``tadm_pages_fork``);
3. each branch appends blocks of tokens: pages are reserved, the block's keys and values stored, and its rows attend over
   the cache, bidirectionally within the block (``tadm_page_attention``);
4. all branches but the first of each prompt are freed and the pool is compacted (``tadm_pages_free``,
   ``tadm_pages_compact``); the survivors go on, one token at a time, drawn from the logits of their last rows with
   settings of their own (``tadm_sample``).

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

    def __init__(self, layers=4, heads=16, kv_heads=8, hd=128, seqs=24, max_len=2048, pages=256, seed=0, check=False,
                 adapters=3, rank=16, vocab=5000):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        d = heads * hd
        rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.wqkv = [(rand((heads + 2 * kv_heads) * hd, d) / math.sqrt(d)).bfloat16() for _ in range(layers)]
        self.wo = [(rand(d, d) / math.sqrt(d)).bfloat16() for _ in range(layers)]
        lora = lambda n_out, n_in: [((rand(adapters, rank, n_in) / math.sqrt(n_in)).bfloat16(),  # noqa: E731
                                     (0.1 * rand(adapters, n_out, rank) / math.sqrt(rank)).bfloat16()) for _ in range(layers)]
        self.lora_qkv, self.lora_o = lora((heads + 2 * kv_heads) * hd, d), lora(d, d)
        self.lora_scale = torch.ones(adapters, device="cuda")
        self.adapter = torch.full((seqs,), -1, dtype=torch.int32, device="cuda")      # of each sequence
        self.gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
        self.embed = rand(vocab, d).bfloat16()                                        # the output head, too
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
    def lora(self, x, w, ab, cu, adapter, dtype=torch.bfloat16):
        y = torch.empty((x.shape[0], w.shape[0]), dtype=dtype, device="cuda")
        a, b = ab
        need = T.tadm_lora_scratch_size(cu.numel() - 1, *x.shape, w.shape[0], a.shape[0], a.shape[1], 1)
        T.tadm_lora_project(x, w, y, cu, adapter, a, b, self.lora_scale, torch.empty(need, dtype=torch.uint8, device="cuda"))
        return y

    def project(self, n, layer, cu, adapter):
        qkv = self.lora(n, self.wqkv[layer], self.lora_qkv[layer], cu, adapter)
        qkv = qkv.view(n.shape[0], self.heads + 2 * self.kv_heads, self.hd)
        return qkv[:, :self.heads], qkv[:, self.heads:self.heads + self.kv_heads], qkv[:, self.heads + self.kv_heads:]

    def begin(self, x):
        """The residual stream (a copy of x) and its norm."""
        n = torch.empty(x.shape, dtype=torch.bfloat16, device="cuda")
        h = torch.empty_like(x)
        T.tadm_residual_norm(x, x, h, n, pre_gain=self.gain, residual_scale=0.0)
        return h, n

    def output(self, h, n, o, layer, cu, adapter):
        """Adds the attention's projection to the stream h and leaves the norm of that in n."""
        y = self.lora(o.view(h.shape[0], -1), self.wo[layer], self.lora_o[layer], cu, adapter, torch.float32)
        T.tadm_residual_norm(h, y, h, n, pre_gain=self.gain)

    def draw(self, n, u, **settings):
        """A token per row of normalised states, from the random numbers u."""
        logits = torch.empty((n.shape[0], self.embed.shape[0]), dtype=torch.float32, device="cuda")
        T.tadm_gemm(n, self.embed, logits, dtype=1)
        tok = torch.empty(n.shape[0], dtype=torch.int32, device="cuda")
        T.tadm_sample(logits, u, tok, **settings)
        return tok

    def prefill(self, x, seqs, lens):
        """Whole prompts, packed: x fp32 [sum(lens), d]; they become tokens 0 .. of the (empty) sequences seqs."""
        self.reserve(seqs, lens)
        cu, start = self.ints(_cum(lens)), self.ints([0] * len(lens))
        table = self.tables[self.ints(seqs).long()].contiguous()
        adapter = self.adapter[self.ints(seqs).long()].contiguous()
        h, n = self.begin(x)
        for layer in range(self.layers):
            q, k, v = self.project(n, layer, cu, adapter)
            o = torch.empty((x.shape[0], self.heads, self.hd), dtype=torch.bfloat16, device="cuda")
            T.tadm_attention_packed(q, k, v, o, cu, max(lens))
            T.tadm_page_write(self.pool, layer, k, v, cu, start, table, max(lens))
            self.output(h, n, o, layer, cu, adapter)
        self.lens[self.ints(seqs).long()] = self.ints(lens)
        return h, n

    def step(self, x, seqs, rows, causal=False):
        """`rows` new tokens of every sequence of seqs: x fp32 [len(seqs) * rows, d].  The final stream and its norm."""
        at = self.ints(seqs).long()
        old = self.lens[at].tolist()
        new = [n + rows for n in old]
        self.reserve(seqs, new)
        table, cu = self.tables[at].contiguous(), self.ints(_cum([rows] * len(seqs)))
        start, lens = self.ints(old), self.ints(new)
        need = T.tadm_page_attention_scratch_size(len(seqs), x.shape[0], rows, max(new), self.heads, self.kv_heads, self.hd, 1)
        scratch = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        adapter = self.adapter[at].contiguous()
        h, n = self.begin(x)
        for layer in range(self.layers):
            q, k, v = self.project(n, layer, cu, adapter)
            o = torch.empty((x.shape[0], self.heads, self.hd), dtype=torch.bfloat16, device="cuda")
            T.tadm_page_write(self.pool, layer, k, v, cu, start, table, rows)
            T.tadm_page_attention(q, self.pool, layer, o, cu, lens, table, rows, max(new), scratch, causal=causal)
            if self.check:
                self.compare(q, o, layer, table, new, rows, causal)
            self.output(h, n, o, layer, cu, adapter)
        self.lens[at] = lens
        return h, n

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
    s.adapter[:] = s.ints(i % prompts % 4 - 1 for i in range(prompts * branches))     # none, and three of them; a prompt's for its branches
    s.prefill(rand(sum(lens)), first, lens)
    others = list(range(prompts, prompts * branches))
    s.fork([i % prompts for i in others], others)
    every = first + others
    for _ in range(blocks):
        x, n = s.step(rand(len(every) * block), every, block)
    peak = int((s.refs > 0).sum())
    s.free(others)
    live = s.compact()
    settings = dict(temperature=torch.linspace(0.0, 1.2, prompts).cuda(), top_p=torch.full((prompts,), 0.9).cuda(),
                    top_k=s.ints(40 if i % 2 else 0 for i in first))
    n = n.view(len(every), block, -1)[:prompts, -1]           # the last row of each survivor
    for _ in range(tokens):
        tok = s.draw(n, torch.rand(prompts, generator=g).cuda(), **settings)
        x, n = s.step(s.embed[tok.long()].float(), first, 1, causal=True)
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
