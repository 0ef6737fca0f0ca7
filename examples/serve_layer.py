"""One decoder layer as a server runs it: prompts of unequal lengths, then single tokens, every projection obfuscated.

    H = norm(residual + X)                       gelo_rms_norm
    Z = H W_qkv     through A, shields, A^-1     gelo_qkv_forward
    Q, cache <- rotated Z                        gelo_rope_append
    O = attention over the cache                 gelo_attention
    X' = O W_o      with an A of its own         gelo_qkv_forward

    python examples/serve_layer.py [--seqs 4] [--prompt 200] [--steps 8] [--dtype bf16]

Prints the time of the prompts and of a step, and how far the layer's results are from the same layer in float64 on the
plain weights (the obfuscation cancels out: Z equals H W_qkv)."""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_05035_amd import binding as g  # noqa: E402

EPS = 1e-5


class Pages:
    """A paged cache and who owns which of its pages; pages are taken from the end of a free list as sequences grow."""

    def __init__(self, n_seqs, max_len, heads, page_rows, width, dtype):
        each = (max_len + page_rows - 1) // page_rows
        shape = (n_seqs * each, heads, page_rows, width)
        self.K, self.V = (torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(2))
        self.cache = g.KvCache(self.K, self.V)
        self.free, self.page_rows, self.max_len = list(range(shape[0])), page_rows, max_len
        self.table = torch.zeros((n_seqs, each), dtype=torch.int32)
        self.length = [0] * n_seqs

    def grow(self, rows):
        """`rows` more rows for each sequence; returns the description of that batch."""
        for s, n in enumerate(rows):
            for p in range((self.length[s] + self.page_rows - 1) // self.page_rows, (self.length[s] + n + self.page_rows - 1) // self.page_rows):
                self.table[s, p] = self.free.pop()
            self.length[s] += n
        start = None
        if any(n != 1 for n in rows):
            start = torch.tensor([sum(rows[:i]) for i in range(len(rows) + 1)], dtype=torch.int32).cuda()
        return g.SeqBatch(torch.tensor(self.length, dtype=torch.int32).cuda(), self.table.cuda(), self.max_len, row_start=start, max_rows=max(rows))


class Layer:
    def __init__(self, ctx, d, q_heads, kv_heads, width, max_len, dtype, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
        self.ctx, self.d, self.q_heads, self.kv_heads, self.width, self.dtype = ctx, d, q_heads, kv_heads, width, dtype
        self.gamma = (1 + 0.1 * rand(d)).to(dtype)
        self.W_qkv = (0.02 * rand(d, (q_heads + 2 * kv_heads) * width)).to(dtype)
        self.W_o = (0.02 * rand(q_heads * width, d)).to(dtype)
        self.table = g.gelo_rope_table(ctx, width, max_len)
        self.batch_id = 0
        g.gelo_reserve_attention(ctx, width)

    def project(self, H, W):
        """H W through the protocol, with a fresh orthogonal A and 5% shield rows."""
        Z = torch.empty((H.shape[0], W.shape[1]), dtype=self.dtype, device="cuda")
        g.gelo_qkv_forward(self.ctx, g.GELO_ORTHOGONAL, H, W, Z, k_shield=max(1, round(0.05 * H.shape[0])), batch_id=self.batch_id)
        self.batch_id += 1
        return Z

    def forward(self, X, residual, pages, batch):
        """(the layer's output, the residual stream it is to be added to)"""
        H, stream = torch.empty_like(X), torch.empty_like(X)
        g.gelo_rms_norm(self.ctx, X, self.gamma, EPS, H=H, residual=residual, residual_out=stream)
        Z = self.project(H, self.W_qkv)
        Q = Z[:, :self.q_heads * self.width]                 # the queries turn where they lie
        g.gelo_rope_append(self.ctx, Z, self.q_heads, pages.cache, batch, Q=Q, table=self.table, rot_dim=self.width)
        O = torch.empty((X.shape[0], self.q_heads * self.width), dtype=self.dtype, device="cuda")
        g.gelo_attention(self.ctx, Q, O, self.q_heads, pages.cache, batch, 1 / math.sqrt(self.width))
        return self.project(O, self.W_o), stream

    def exact(self, X, residual):
        """The same layer for one whole sequence in float64, without cache or obfuscation."""
        n, w = X.shape[0], self.width
        h = X.double() + residual.double()
        H = h / (h.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * self.gamma.double()
        z = (H @ self.W_qkv.double()).view(n, -1, w)
        angle = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, w, 2, device="cuda", dtype=torch.float64) / w)
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        a, b = z[..., :w // 2], z[..., w // 2:]
        turned = torch.cat((a * c - b * s, b * c + a * s), -1)
        q, k, v = turned[:, :self.q_heads], turned[:, self.q_heads:self.q_heads + self.kv_heads], z[:, self.q_heads + self.kv_heads:]
        k, v = (x.repeat_interleave(self.q_heads // self.kv_heads, 1) for x in (k, v))
        hidden = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
        score = (torch.einsum("ihw,jhw->hij", q, k) / math.sqrt(w)).masked_fill(hidden, -math.inf)
        return torch.einsum("hij,jhw->ihw", torch.softmax(score, -1), v).reshape(n, -1) @ self.W_o.double()


def serve(seqs=4, prompt=200, steps=8, dtype=torch.bfloat16, d=1024, q_heads=16, kv_heads=4, width=64, page_rows=16):
    """Runs prompts and steps; returns (relative error over all rows, seconds of the prompts, seconds of a step)."""
    ctx = g.gelo_create(0, 1234)
    try:
        lens = [max(1, prompt - 37 * s) for s in range(seqs)]
        max_len = max(lens) + steps
        layer = Layer(ctx, d, q_heads, kv_heads, width, max_len, dtype)
        pages = Pages(seqs, max_len, kv_heads, page_rows, width, dtype)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(1)
        X, R = ([torch.randn((n + steps, d), generator=gen, device="cuda").to(dtype) for n in lens] for _ in range(2))
        got = [[] for _ in range(seqs)]
        times = []
        for step in range(steps + 1):
            rows = lens if step == 0 else [1] * seqs
            at = [(0, n) if step == 0 else (n + step - 1, n + step) for n in lens]
            batch = pages.grow(rows)
            x, r = (torch.cat([t[a:b] for t, (a, b) in zip(T, at)]) for T in (X, R))
            torch.cuda.synchronize()
            began = time.perf_counter()
            out, _ = layer.forward(x, r, pages, batch)
            torch.cuda.synchronize()
            times.append(time.perf_counter() - began)
            for s, part in enumerate(out.split(rows)):
                got[s].append(part)
        far = size = 0.0
        for s in range(seqs):
            want = layer.exact(X[s], R[s])
            far += float((torch.cat(got[s]).double() - want).pow(2).sum())
            size += float(want.pow(2).sum())
        return math.sqrt(far / size), times[0], sorted(times[1:])[steps // 2] if steps else 0.0
    finally:
        g.gelo_destroy(ctx)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--seqs", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=200)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args()
    error, first, step = serve(a.seqs, a.prompt, a.steps, torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    print(f"prompts {first * 1e3:.2f} ms (first use), a step {step * 1e6:.0f} us, relative error {error:.2e}")


if __name__ == "__main__":
    main()
