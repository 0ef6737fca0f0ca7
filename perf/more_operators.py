"""What a server of many tenants adds around an obfuscated projection, as cases for timing: every request's own low-rank adapter
beside the shared weight, and a paged cache that holds keys and values in 4 bits, filled with rotated rows and read by attention.

  own                   False: run() computes the operators in their plain form, True: by this library's entry points
  listed()              the cases
  draw(rng)             one more case of the same ranges
  prepare(case, seed)   what a program holds before the call: activations, adapters, the cache and who owns which of its pages
  run(state)            one pass through an operator; its outputs
  work(case)            bytes and operations one pass cannot do without
  exact(case, seed)     the outputs in 64 bits

Cases by "op":
  adapt    Z[i] = base[i] + scale[w] (H[i] A[w]^T) B[w]^T, w the adapter of row i; a fused projection's parts have an A each
  append4  rotate the queries and keys of a fused Q|K|V row, put keys and values, 4 bits each, into the pages of the row's sequence
  attend4  softmax(scale q k^T) v over the sequence's rows of that cache, up to the query's own row or (cross) over all

A block of 32 values of a head is held as codes of 4 bits (sign; 0, 0.5, 1, 1.5, 2, 3, 4, 6) times 2^e, e the least whole number from -110 to 125
with max |value| <= 7 2^e, rounded to nearest, ties to the even code; e + 127 is the block's scale byte.  A head's piece of a page is its rows' codes, two
to a byte, then their scale bytes.  Of keys row by row; of values four rows at a time: of each row's D / 2 bytes of codes in 16 pieces (of each row's
scale bytes) the first of the four rows, then the second of the four rows, ...
"""
import math
import random

import torch

own = False

ROPE_BASE = 10000.0
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _adapt(name, dtype, n, d, parts, rank, n_adapters, order, without):
    """parts: widths of the projection's parts; order: rows of one adapter side by side ("runs") or anywhere ("any"); without: part of the rows without one."""
    c = {"op": "adapt", "dtype": dtype, "n": n, "d": d, "parts": "+".join(str(p) for p in parts), "rank": rank, "n_adapters": n_adapters, "order": order,
         "without": without}
    return dict(c, name=name) if name else c


def _seqs(name, op, dtype, n_seqs, new, past, heads, d, page, rot=0, layout="half", causal=True):
    """`new` and `past`: the fewest and the most rows that a sequence brings and has in the cache already."""
    c = {"op": op, "dtype": dtype, "n_seqs": n_seqs, "new_min": new[0], "new_max": new[1], "past_min": past[0], "past_max": past[1],
         "hq": heads[0], "hkv": heads[1], "d": d, "page": page, "rot": rot, "layout": layout, "causal": causal}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest batch there is: three requests, two adapters, a narrow model in float
        _adapt("adapt_tiny_f32", "f32", 3, 768, (768, 768, 768), 8, 2, "any", 0.0),
        # a decode step of the 4096-wide model: 64 requests draw on 48 adapters, some of them on none
        _adapt("adapt_decode", "bf16", 64, 4096, (4096, 4096, 4096), 16, 48, "any", 0.1),
        # prompts: 8 sequences x 512 tokens, each with an adapter of its own, beside the fused projection
        _adapt("adapt_prompts", "bf16", 4096, 4096, (4096, 4096, 4096), 16, 8, "runs", 0.0),
        # the output projection of a prefill batch with one wide adapter
        _adapt("adapt_wide", "bf16", 2048, 4096, (4096,), 64, 1, "runs", 0.0),
        # one token of each of 64 sequences goes into the cache
        _seqs("append4_decode", "append4", "bf16", 64, (1, 1), (100, 255), (32, 32), 128, 16, rot=128),
        # prompts of unequal lengths, grouped heads, half of each head rotated in interleaved pairs
        _seqs("append4_prompts", "append4", "bf16", 8, (301, 512), (0, 0), (32, 8), 128, 64, rot=64, layout="pairs"),
        # three young sequences in float
        _seqs("decode4_tiny_f32", "attend4", "f32", 3, (1, 1), (0, 199), (6, 2), 64, 16),
        # the decode step behind the sweep's prompts: 64 sequences of some hundred tokens, a key head to every query head
        _seqs("decode4_step", "attend4", "bf16", 64, (1, 1), (400, 639), (32, 32), 128, 16),
        # few long sequences with grouped heads: the cache's length has to be split to fill the chip
        _seqs("decode4_long", "attend4", "bf16", 3, (1, 1), (20000, 32767), (32, 8), 128, 64),
        # a full serving batch at the 4096 tokens of the model: memory bandwidth
        _seqs("decode4_full", "attend4", "bf16", 64, (1, 1), (3500, 4095), (32, 32), 128, 64),
        # the prompts of the sweep, of unequal lengths
        _seqs("prompts4", "attend4", "bf16", 8, (301, 512), (0, 0), (32, 32), 128, 16),
        # a long prompt's next part behind rows that are in the cache already, grouped heads: the matrix cores
        _seqs("prompt4_long", "attend4", "bf16", 1, (6000, 6000), (2000, 2000), (32, 8), 128, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(32, 32), (32, 8), (8, 8), (28, 4), (14, 2), (64, 8), (16, 1), (5, 5), (48, 2)]


def draw(rng):
    """One more case: rows, widths, ranks, adapters, lengths, head layouts, page sizes and types over their ranges."""
    op = rng.choice(["adapt", "adapt", "adapt", "append4", "append4", "decode", "decode", "decode", "prompt", "prompt", "cross"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    size = 2 if dtype == "f32" else 1
    if op == "adapt":
        d = 8 * max(1, round(_log_int(rng, 64, 8192) / 8))
        wide, narrow = (16 * max(1, round(_log_int(rng, 64, 8192) / 16)) for _ in range(2))
        parts = rng.choice([(wide,), (wide, narrow), (wide, narrow, narrow), (wide, wide, wide)])
        rank, adapters = rng.choice([8, 16, 16, 32, 64, 128]), _log_int(rng, 1, 64)
        each = rank * (d * len(parts) + sum(parts))                                     # values of an adapter
        adapters = max(1, min(adapters, (1 << 26) // each))
        most = 4096 * (4096 + 2 * 12288) // (size * (d + 2 * sum(parts) + 2 * rank * len(parts) * adapters))       # rows of the largest listed case's memory
        n = min(_log_int(rng, 1, 8192), max(1, most), max(1, (1 << 32) // (size * each)))
        return _adapt(None, dtype, n, d, parts, rank, adapters, rng.choice(["runs", "any"]), rng.choice([0.0, 0.0, 0.2]))
    heads, d, page = rng.choice(HEADS), rng.choice([64, 96, 128, 128, 256]), rng.choice([16, 32, 64, 128])
    if op == "append4":
        new = _log_int(rng, 1, 1024)
        seqs = max(1, min(_log_int(rng, 1, 128), 4096 * 8192 // (new * (heads[0] + 2 * heads[1]) * d)))
        past = rng.choice([0, _log_int(rng, 1, 256)])
        rot = rng.choice([d, d, d // 2])
        return _seqs(None, "append4", dtype, seqs, (max(1, new // 2), new), (past // 2, past), heads, d, page, rot, rng.choice(["half", "half", "pairs"]))
    if op == "decode":
        most = 64 * 4096 * 32 * 128 // (heads[1] * d * size)          # rows of the cache in all
        past = min(_log_int(rng, 1, 65536), most - 1)
        seqs = max(1, min(_log_int(rng, 1, 128), most // (past + 1)))
        return _seqs(None, "attend4", dtype, seqs, (1, 1), (past // 2, past), heads, d, page)
    new = _log_int(rng, 2, 6000)
    past = _log_int(rng, 1, 2000) if op == "cross" else rng.choice([0, _log_int(rng, 1, 2000)])
    rows = past if op == "cross" else past + new
    pairs = 32 * 6000 * 8000 * 128 // (size * size * size)
    while new > 2 and heads[0] * d * new * rows > pairs:
        new, rows = new // 2, rows if op == "cross" else past + new // 2
    seqs = max(1, min(_log_int(rng, 1, 16), pairs // (heads[0] * d * new * rows)))
    return _seqs(None, "attend4", dtype, seqs, (max(1, new // 2), new), (max(1, past // 2) if op == "cross" else past // 2, past), heads, d, page,
                 causal=op != "cross")


def _parts(case):
    return [int(p) for p in case["parts"].split("+")]


def _lengths(case):
    """(new rows, rows of the cache to attend to) of every sequence: the longest first, the others anywhere in the range."""
    rng = random.Random(case["n_seqs"] * 1000003 + case["past_max"] * 1009 + case["new_max"])
    new, kv = [], []
    for i in range(case["n_seqs"]):
        n = case["new_max"] if i == 0 else rng.randint(case["new_min"], case["new_max"])
        past = case["past_max"] if i == 0 else rng.randint(case["past_min"], case["past_max"])
        new.append(n)
        kv.append(past + n if case["causal"] else past)
    return new, kv


class _State:
    """Inputs and outputs of one case, and what a program keeps beside them."""

    handles = None


def _which(case):
    """The adapter of each row, -1 for none."""
    rng = random.Random(case["n"] * 1000003 + case["n_adapters"] * 1009 + case["rank"])
    n, count = case["n"], case["n_adapters"]
    at = [i * count // n if case["order"] == "runs" else rng.randrange(count) for i in range(n)]
    return [-1 if rng.random() < case["without"] else w for w in at]


def _pack(x, values):
    """A head's pieces of pages from their rows: (pages, heads, rows, width) float -> (pages, heads, bytes)."""
    pages, heads, rows, d = x.shape
    blocks = x.view(pages, heads, rows, d // 32, 32)
    f, k = torch.frexp(blocks.abs().amax(-1))
    e = torch.where(f <= 0.875, k - 3, k - 2).clamp(-110, 125)
    y = torch.ldexp(blocks.abs(), -e[..., None])
    codes = torch.where(y < 2, (2 * y).round(), torch.where(y < 4, y.round() + 2, (y / 2).round() + 4)).clamp(max=7).to(torch.uint8)
    codes = (codes | (torch.signbit(blocks).to(torch.uint8) << 3)).view(pages, heads, rows, d // 2, 2)
    codes, scales = codes[..., 0] | (codes[..., 1] << 4), (e + 127).to(torch.uint8)
    if values:
        codes = codes.view(pages, heads, rows // 4, 4, 16, d // 32).transpose(3, 4)
        scales = scales.view(pages, heads, rows // 4, 4, d // 32).transpose(3, 4)
    return torch.cat((codes.reshape(pages, heads, -1), scales.reshape(pages, heads, -1)), -1)


def prepare(case, seed):
    s = _State()
    s.case = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    if case["op"] == "adapt":
        n, d, rank, count = case["n"], case["d"], case["rank"], case["n_adapters"]
        s.ends, p = [], 0
        for part in _parts(case):
            p += part
            s.ends.append(p)
        # eight channels of twenty times the scale, as the activations of language models have them
        s.H = normal(n, d)
        s.H[:, torch.randperm(d, generator=gen, device="cuda")[:8]] *= 20.0
        s.H = s.H.to(dtype)
        s.A = (normal(count, len(s.ends) * rank, d) / math.sqrt(d)).to(dtype)
        s.B = (0.1 * normal(count, p, rank)).to(dtype)
        s.scale = 0.5 + 1.5 * torch.rand(count, generator=gen, device="cuda")
        s.which = torch.tensor(_which(case), dtype=torch.int32, device="cuda")
        s.base = normal(n, p).to(dtype)
        s.Z = torch.empty_like(s.base)
        return s
    new, kv = _lengths(case)
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    s.n_rows, s.max_rows, s.max_kv = sum(new), max(new), max(kv)
    pages = [(x + page - 1) // page for x in kv]
    total = sum(pages) + 3
    s.K, s.V = (torch.empty((total, hkv, page * d * 17 // 32), dtype=torch.uint8, device="cuda") for _ in range(2))
    at_once = max(1, (1 << 26) // (hkv * page * d))
    for first in range(0, total, at_once):
        count = min(at_once, total - first)
        # keys have a few channels of a larger scale in every head
        keys = normal(count, hkv, page, d)
        keys[..., 5::41] *= 4.0
        s.K[first:first + count] = _pack(keys, False)
        s.V[first:first + count] = _pack(normal(count, hkv, page, d), True)
    # the pages of a sequence lie anywhere in the cache
    free = torch.randperm(total, generator=gen, device="cuda").int()
    first = torch.tensor([sum(pages[:i]) for i in range(len(pages))], device="cuda")
    at = torch.arange(max(pages), device="cuda")
    count = torch.tensor(pages, device="cuda")
    s.table = torch.where(at < count[:, None], free[(first[:, None] + at).clamp(max=sum(pages))], torch.zeros((), dtype=torch.int32, device="cuda"))
    s.kv_len = torch.tensor(kv, dtype=torch.int32, device="cuda")
    s.row_start = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    s.Q = normal(s.n_rows, hq * d).to(dtype)
    if case["op"] == "append4":
        s.QKV = (1.3 * normal(s.n_rows, (hq + 2 * hkv) * d)).to(dtype)
        turn = torch.arange(s.max_kv, device="cuda", dtype=torch.float64)[:, None] * ROPE_BASE ** (
            -torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])
        s.cos_sin = torch.stack((turn.cos(), turn.sin()), -1).float()
        s.new_K, s.new_V = (torch.empty((s.n_rows, hkv * d), dtype=dtype, device="cuda") for _ in range(2))
    s.O = torch.empty((s.n_rows, hq * d), dtype=dtype, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms --
def _plain_adapt(s):
    c = s.case
    n, d, rank, count, parts = c["n"], c["d"], c["rank"], c["n_adapters"], len(s.ends)
    # every row with every adapter, then those that are not the row's out
    t = torch.matmul(s.H.float(), s.A.float().view(-1, d).t().contiguous()).view(n, count, parts, rank)
    t = torch.where((s.which[:, None] == torch.arange(count, device="cuda"))[:, :, None, None], t * s.scale[None, :, None, None], torch.zeros((), device="cuda"))
    part = torch.bucketize(torch.arange(s.ends[-1], device="cuda"), torch.tensor(s.ends, device="cuda"), right=True)
    b = s.B.float()
    wide = torch.where(part[None, :, None, None] == torch.arange(parts, device="cuda")[:, None], b[:, :, None, :], torch.zeros((), device="cuda"))
    wide = wide.permute(0, 2, 3, 1).reshape(count * parts * rank, -1).contiguous()         # adapters, parts, rank x columns
    return {"Z": (s.base.float() + torch.matmul(t.view(n, -1), wide)).to(s.base.dtype)}


def _row_owner(s):
    """Of every new row: its sequence, its number in there, its position in the sequence."""
    row = torch.arange(s.n_rows, device="cuda")
    seq = torch.searchsorted(s.row_start[1:].contiguous(), row.int(), right=True)
    i = row - s.row_start[seq]
    return seq, i, s.kv_len[seq] - (s.row_start[seq + 1] - s.row_start[seq]) + i


def _plain_rotate(x, cos_sin, layout):
    """x: rows, heads, width; cos_sin: rows, rot / 2, 2."""
    rot = 2 * cos_sin.shape[1]
    c, t = cos_sin[:, None, :, 0], cos_sin[:, None, :, 1]
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * c - b * t, b * c + a * t), -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * c - b * t, b * c + a * t), -1).flatten(-2)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_codes(x):
    """(rows, heads, width) -> (bytes of two codes, scale bytes), in x's precision: 64 bits where values next to a border matter."""
    blocks = x.reshape(*x.shape[:2], -1, 32)
    f, k = torch.frexp(blocks.abs().amax(-1))
    e = torch.where(f <= 0.875, k - 3, k - 2).clamp(-110, 125)
    y = torch.ldexp(blocks.abs(), -e[..., None])
    codes = torch.where(y < 2, (2 * y).round(), torch.where(y < 4, y.round() + 2, (y / 2).round() + 4)).clamp(max=7).to(torch.uint8)
    codes = (codes | (torch.signbit(blocks).to(torch.uint8) << 3)).view(*x.shape[:2], -1, 2)
    return codes[..., 0] | (codes[..., 1] << 4), (e + 127).to(torch.uint8)


def _plain_regions(pool, page, d, values):
    """Views of the codes and scale bytes of (..., bytes) pieces by row: (..., rows / 4, 4, 16, D / 32) and (..., rows / 4, 4, D / 32)."""
    codes, scales = pool[..., :page * d // 2], pool[..., page * d // 2:]
    if values:
        return codes.unflatten(-1, (page // 4, 16, 4, d // 32)).transpose(-3, -2), scales.unflatten(-1, (page // 4, d // 32, 4)).transpose(-2, -1)
    return codes.unflatten(-1, (page // 4, 4, 16, d // 32)), scales.unflatten(-1, (page // 4, 4, d // 32))


def _plain_values(codes, scales):
    """(..., D / 2) bytes and (..., D / 32) scale bytes -> (..., D) float."""
    level = torch.tensor(LEVELS + [-x for x in LEVELS], device="cuda")
    pair = torch.stack((level.repeat(16), level.repeat_interleave(16)), -1)                # of every byte
    x = pair[codes.int()].unflatten(-2, (-1, 16)).flatten(-2)                              # ..., blocks, 32
    return torch.ldexp(x, scales.int()[..., None] - 127).flatten(-2)


def _plain_append(s):
    c = s.case
    hq, hkv, d, page = c["hq"], c["hkv"], c["d"], c["page"]
    seq, _, pos = _row_owner(s)
    pos = pos.long()
    x = s.QKV.view(s.n_rows, hq + 2 * hkv, d)
    Q = _plain_rotate(x[:, :hq].float(), s.cos_sin[pos], c["layout"]).to(s.QKV.dtype)
    keys = _plain_rotate(x[:, hq:hq + hkv].double(), s.cos_sin[pos].double(), c["layout"])
    at, slot = s.table[seq, pos // page].long(), pos % page
    out = {"Q": Q.reshape(s.n_rows, hq * d)}
    for name, pool, rows, values in (("K", s.K, keys, False), ("V", s.V, x[:, hq + hkv:].double(), True)):
        codes, scales = _plain_regions(pool, page, d, values)
        new_codes, new_scales = _plain_codes(rows)
        codes[at, :, slot // 4, slot % 4] = new_codes.unflatten(-1, (16, d // 32))
        scales[at, :, slot // 4, slot % 4] = new_scales
        held = _plain_values(codes[at, :, slot // 4, slot % 4].flatten(-2), scales[at, :, slot // 4, slot % 4])
        out[name] = held.reshape(s.n_rows, hkv * d).to(s.QKV.dtype)
    return out


def _plain_attend(s):
    c = s.case
    n_seqs, hq, hkv, d, page = c["n_seqs"], c["hq"], c["hkv"], c["d"], c["page"]
    seq, i, _ = _row_owner(s)
    rows = (s.row_start[:-1, None] + torch.arange(s.max_rows, device="cuda")).clamp(max=s.n_rows - 1)
    q = s.Q.float().view(s.n_rows, hkv, hq // hkv, d)[rows]                             # sequences, rows, key heads, heads, width
    q = q.permute(0, 2, 1, 3, 4).reshape(n_seqs, hkv, s.max_rows * (hq // hkv), d)

    def held(pool, values):
        codes, scales = _plain_regions(pool[s.table.long()].transpose(1, 2), page, d, values)    # sequences, heads, pages of the sequence, ...
        x = _plain_values(codes.flatten(-2).reshape(n_seqs, hkv, -1, d // 2)[:, :, :s.max_kv], scales.reshape(n_seqs, hkv, -1, d // 32)[:, :, :s.max_kv])
        return x.contiguous()

    p = torch.matmul(q, held(s.K, False).transpose(2, 3).contiguous()).view(n_seqs, hkv, s.max_rows, hq // hkv, s.max_kv) * (1.0 / math.sqrt(d))
    last = s.kv_len - (s.row_start[1:] - s.row_start[:-1]) if c["causal"] else s.kv_len - 1
    last = last[:, None] + (torch.arange(s.max_rows, device="cuda") if c["causal"] else torch.zeros(s.max_rows, dtype=torch.int32, device="cuda"))
    hidden = torch.arange(s.max_kv, device="cuda") > last[..., None].clamp(max=s.max_kv)      # sequences, rows, keys
    p.masked_fill_(hidden[:, None, :, None, :], -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n_seqs, hkv, -1, s.max_kv), held(s.V, True)).view(n_seqs, hkv, s.max_rows, hq // hkv, d)
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    return {"O": o.permute(0, 2, 1, 3, 4)[seq, i].reshape(s.n_rows, hq * d).to(s.Q.dtype)}


# --------------------------------------------------------------------------------------------- this library's --
_kept = {}


def _library():
    """The binding and a context of the process, as a serving program keeps them."""
    if not _kept:
        from paper_2603_05035_amd import binding
        _kept["g"], _kept["ctx"] = binding, binding.gelo_create(torch.cuda.current_device(), 1)
    return _kept["g"], _kept["ctx"]


def _own(s):
    g, ctx = _library()
    c = s.case
    if c["op"] == "adapt":
        if s.handles is None:
            s.handles = g.Adapters(s.A, s.B, scale=s.scale, part_ends=s.ends)      # stays as long as the adapters do
        g.gelo_adapt(ctx, s.H, s.handles, s.which, s.Z, base=s.base)
        return {"Z": s.Z}
    if s.handles is None:
        # the descriptions of the cache and of the batch stay as long as their tensors do
        s.handles = (g.KvCacheFp4(s.K, s.V, c["page"], c["d"]),
                     g.SeqBatch(s.kv_len, s.table, s.max_kv, row_start=None if s.max_rows == 1 else s.row_start, max_rows=s.max_rows))
    cache, batch = s.handles
    if c["op"] == "append4":
        g.gelo_rope_append_fp4(ctx, s.QKV, c["hq"], cache, batch, Q=s.O, table=s.cos_sin, rot_dim=c["rot"],
                               layout=g.GELO_ROPE_HALF if c["layout"] == "half" else g.GELO_ROPE_PAIRS)
        g.gelo_cache_rows_fp4(ctx, cache, batch, s.new_K, s.new_V)                # what the new rows are held as
        return {"Q": s.O, "K": s.new_K, "V": s.new_V}
    g.gelo_attention_fp4(ctx, s.Q, s.O, c["hq"], cache, batch, 1.0 / math.sqrt(c["d"]), causal=c["causal"])
    return {"O": s.O}


def run(s):
    if own:
        return _own(s)
    return {"adapt": _plain_adapt, "append4": _plain_append, "attend4": _plain_attend}[s.case["op"]](s)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "adapt":
        n, d, rank, parts = case["n"], case["d"], case["rank"], _parts(case)
        which = [w for w in _which(case) if w >= 0]
        used, p = len(set(which)), sum(parts)
        adapter = rank * (d * len(parts) + p)
        return {"bytes": size * (len(which) * d + 2 * n * p + used * adapter), "flops": 2 * len(which) * adapter}
    new, kv = _lengths(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    rows = sum(new)
    if case["op"] == "append4":
        # into the cache and, for the values that the new rows are held as, out of it
        return {"bytes": rows * ((2 * hq + 2 * hkv) * d * size + case["rot"] * 4 + 2 * hkv * d * 17 // 32 + 2 * hkv * d * size), "flops": 3 * rows * (hq + hkv) * case["rot"]}
    seen = sum(n * x - n * (n - 1) // 2 if case["causal"] else n * x for n, x in zip(new, kv))      # pairs of a query and a key
    return {"bytes": 2 * rows * hq * d * size + 2 * sum(kv) * hkv * d * 17 // 32, "flops": 4 * hq * d * seen}


# ------------------------------------------------------------------------------------------------- in 64 bits --
def _exact_held(x):
    """What (..., D) doubles are held as: by the distances to the levels' middles."""
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    top = blocks.abs().max(-1, keepdim=True).values
    e = torch.log2(top / 7).ceil()
    e = torch.where(top <= 7 * torch.exp2(e - 1), e - 1, torch.where(top > 7 * torch.exp2(e), e + 1, e)).clamp(-110, 125)
    y = blocks.abs() / torch.exp2(e)
    code = torch.zeros_like(y, dtype=torch.int64)
    for k in range(7):                                       # above the middle of two levels, or on it where the upper one is the even code
        middle = (LEVELS[k] + LEVELS[k + 1]) / 2
        code += y >= middle if k % 2 else y > middle
    held = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")[code] * torch.exp2(e)
    return torch.where(blocks < 0, -held, held).reshape(x.shape)


def _exact_read(piece, rows, d, values):
    """A head's pieces of a sequence's pages -> its rows in double, byte by byte as the layout says."""
    pages, page = piece.shape[0], piece.shape[1] * 32 // 17 // d
    row = torch.arange(rows, device="cuda")
    comp = torch.arange(d, device="cuda")
    in_page, base = row % page, row // page
    if values:
        four, r, u = in_page // 4, in_page % 4, d // 32
        code_at = (four * 2 * d + r * u)[:, None] + (comp // 2 // u * 4 * u + comp // 2 % u)
        scale_at = page * d // 2 + (four * 4 * u + r)[:, None] + 4 * (comp // 32)
    else:
        code_at = (in_page * (d // 2))[:, None] + comp // 2
        scale_at = page * d // 2 + (in_page * (d // 32))[:, None] + comp // 32
    byte = piece[base[:, None], code_at].long()
    code = torch.where(comp % 2 == 1, byte >> 4, byte & 15)
    size = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")[code & 7] * torch.exp2(piece[base[:, None], scale_at].double() - 127)
    return torch.where(code >= 8, -size, size)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adapt":
        Z = s.base.double()
        rank, which = case["rank"], s.which.cpu()
        for w in sorted(set(which.tolist()) - {-1}):
            rows = (which == w).nonzero()[:, 0].cuda()
            begin = 0
            for k, end in enumerate(s.ends):
                t = s.H[rows].double() @ s.A[w, k * rank:(k + 1) * rank].double().T
                Z[rows, begin:end] += float(s.scale[w]) * (t @ s.B[w, begin:end].double().T)
                begin = end
        return {"Z": Z}
    new, kv = _lengths(case)
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    table = s.table.cpu()
    group = hq // hkv
    first = 0
    if case["op"] == "append4":
        Q = torch.empty((s.n_rows, hq, d), dtype=torch.float64, device="cuda")
        K, V = (torch.empty((s.n_rows, hkv, d), dtype=torch.float64, device="cuda") for _ in range(2))
        rot = case["rot"]
        for b in range(case["n_seqs"]):
            x = s.QKV[first:first + new[b]].double().view(new[b], hq + 2 * hkv, d)
            at = torch.arange(kv[b] - new[b], kv[b], device="cuda")
            angles = s.cos_sin[at].double()[:, None]
            part = x[:, :hq + hkv, :rot].reshape(new[b], hq + hkv, rot)
            pairs = part.view(new[b], -1, 2, rot // 2).transpose(2, 3) if case["layout"] == "half" else part.view(new[b], -1, rot // 2, 2)
            cos, sin = angles[..., 0], angles[..., 1]
            turned = torch.stack((pairs[..., 0] * cos - pairs[..., 1] * sin, pairs[..., 0] * sin + pairs[..., 1] * cos), -1)
            turned = turned.transpose(2, 3).reshape(part.shape) if case["layout"] == "half" else turned.reshape(part.shape)
            x[:, :hq + hkv, :rot] = turned
            Q[first:first + new[b]] = x[:, :hq]
            K[first:first + new[b]] = _exact_held(x[:, hq:hq + hkv])
            V[first:first + new[b]] = _exact_held(x[:, hq + hkv:])
            first += new[b]
        return {"Q": Q.view(s.n_rows, hq * d), "K": K.view(s.n_rows, hkv * d), "V": V.view(s.n_rows, hkv * d)}
    O = torch.empty((s.n_rows, hq, d), dtype=torch.float64, device="cuda")
    for b in range(case["n_seqs"]):
        used = table[b, :(kv[b] + page - 1) // page].long().cuda()
        row = torch.arange(new[b], device="cuda")[:, None]
        key = torch.arange(kv[b], device="cuda")
        seen = key <= row + (kv[b] - new[b]) if case["causal"] else torch.ones((new[b], kv[b]), dtype=torch.bool, device="cuda")
        bias = torch.zeros(seen.shape, dtype=torch.float64, device="cuda").masked_fill_(~seen, -math.inf)
        for h in range(hkv):
            k, v = _exact_read(s.K[used, h], kv[b], d, False), _exact_read(s.V[used, h], kv[b], d, True)
            for j in range(h * group, (h + 1) * group):
                q = s.Q[first:first + new[b], j * d:(j + 1) * d].double()
                O[first:first + new[b], j] = torch.softmax(q @ k.T / math.sqrt(d) + bias, -1) @ v
        first += new[b]
    return {"O": O.view(s.n_rows, hq * d)}
