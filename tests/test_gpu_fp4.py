"""The paged cache of 4 bits - append, rows read back, attention - through the C ABI, against the float64 reference.

What is held is compared for equality.  Bounds of attention, element by element, are those of the attention over values, from the formats' unit roundoffs U32 =
2^-24 and U16 = 2^-8 (bfloat16); see attention_bound."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from oracle import serve_oracle as so
from paper_2603_05035_amd import binding as g

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = g.gelo_create(0, 1)
    yield c
    g.gelo_destroy(c)


def host(t):
    return t.double().cpu().numpy()


def rand(shape, seed, dtype, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(shape, generator=gen)).to(dtype).cuda()


def padded(rows, cols, ld, dtype, fill=7.0):
    """A rows x cols view with leading dimension ld, and the whole buffer."""
    whole = torch.full((rows, ld), fill, dtype=dtype, device="cuda")
    return whole[:, :cols], whole


def within(got, want, bound, what=""):
    got = host(got) if isinstance(got, torch.Tensor) else got
    off = np.abs(got - want) - bound
    assert not np.isnan(got).any(), what
    assert off.max() <= 0, (what, float(off.max()), np.unravel_index(off.argmax(), off.shape))


def make_batch(new, kv, page, seed, spare=3, max_kv=None, one_row=False):
    """Pages in random places; entries behind a sequence's last page are poison: they must not be read."""
    pages = [(x + page - 1) // page for x in kv]
    n_pages = sum(pages) + spare
    where = np.random.default_rng(seed).permutation(n_pages)
    max_kv = max_kv or max(max(kv), 1)
    table = np.full((len(kv), (max_kv + page - 1) // page), 1 << 30, dtype=np.int32)
    at = 0
    for s, n in enumerate(pages):
        table[s, :n] = where[at:at + n]
        at += n
    row_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    batch = g.SeqBatch(torch.tensor(kv, dtype=torch.int32).cuda(), torch.from_numpy(table).cuda(), max_kv,
                       row_start=None if one_row else torch.from_numpy(row_start).cuda(), max_rows=max(max(new), 1))
    return batch, table, row_start, n_pages


def pools(n_pages, heads, page, d, fill=0xA5, order="pages"):
    """Keys' and values' bytes; order "heads": the pages of a head side by side, "both": keys and values of a page in one piece of memory, with a gap."""
    piece = so.piece_bytes(page, d)
    if order == "both":
        whole = torch.full((n_pages, 2, heads, piece + 48), fill, dtype=torch.uint8, device="cuda")
        return whole[:, 0, :, :piece], whole[:, 1, :, :piece]
    shape = (heads, n_pages, piece) if order == "heads" else (n_pages, heads, piece)
    K, V = (torch.full(shape, fill, dtype=torch.uint8, device="cuda") for _ in range(2))
    return (K.permute(1, 0, 2), V.permute(1, 0, 2)) if order == "heads" else (K, V)


def filled(n_pages, heads, page, d, seed, order="pages"):
    """Pools that hold N(0, 1), and what they hold in float64."""
    K, V = pools(n_pages, heads, page, d, order=order)
    values = []
    for pool, of_values in ((K, False), (V, True)):
        seed += 1
        codes, scales = so.hold(np.random.default_rng(seed).standard_normal((n_pages, heads, page, d)))
        pool.copy_(torch.from_numpy(so.pack(codes, scales, of_values)))
        values.append(so.held(codes, scales))
    return K, V, *values


# -------------------------------------------------------------------------------------------------------- append --
APPENDS = [  # dtype, new rows, rows in the cache with them, q heads, kv heads, d, page, order, rot, pairs
    (BF16, [1, 1, 1], [1, 16, 17], 4, 4, 64, 16, "pages", 64, False),
    (BF16, [5, 0, 33, 1], [5, 9, 40, 64], 6, 2, 128, 32, "heads", 64, True),
    (F32, [2, 31], [130, 31], 5, 5, 96, 64, "both", 96, False),
    (F32, [17], [20], 2, 1, 256, 16, "pages", 16, True),
    (BF16, [70], [70], 7, 1, 160, 128, "both", 48, False),
    (BF16, [9, 12], [9, 12], 0, 3, 64, 16, "heads", 0, False),
    (F32, [3], [3], 1, 2, 32, 16, "pages", 32, False),
    (BF16, [40, 3], [300, 1003], 8, 8, 256, 16, "pages", 256, False),
    (BF16, [64, 200], [64, 200], 32, 32, 128, 16, "pages", 128, False),
    (F32, [130], [4000], 8, 2, 128, 64, "heads", 128, True),
]


@pytest.mark.parametrize("dtype,new,kv,hq,hkv,d,page,order,rot,pairs", APPENDS)
def test_append_and_rows_read_back(ctx, dtype, new, kv, hq, hkv, d, page, order, rot, pairs):
    """Codes and scale bytes to the bit: a rotation in double is two exact products (of 24 bits each at most) and their sum, rounded at 53 bits whatever the
    order.  Queries to the bit those of the append of values.  No other byte moves.  Rows read back are what is held."""
    batch, table, row_start, n_pages = make_batch(new, kv, page, 1)
    rows = int(row_start[-1])
    K, V = pools(n_pages, hkv, page, d, order=order)
    QKV, _ = padded(rows, (hq + 2 * hkv) * d, (hq + 2 * hkv) * d + 8, dtype)
    QKV.copy_(rand(QKV.shape, 2, dtype))
    Q, Q_all = padded(rows, hq * d, hq * d + 24, dtype) if hq else (None, None)
    cs = g.gelo_rope_table(ctx, rot, max(kv)) if rot else None
    layout = g.GELO_ROPE_PAIRS if pairs else g.GELO_ROPE_HALF
    cache = g.KvCacheFp4(K, V, page, d)
    g.gelo_rope_append_fp4(ctx, QKV, hq, cache, batch, Q=Q, table=cs, rot_dim=rot, layout=layout)
    x = host(QKV).reshape(rows, hq + 2 * hkv, d)
    keys = x[:, hq:hq + hkv].copy()
    first = np.arange(rot // 2) * 2 if pairs else np.arange(rot // 2)
    second = first + 1 if pairs else first + rot // 2
    want = [np.full(K.shape, 0xA5, dtype=np.uint8) for _ in range(2)]
    at_bytes = [so.places(page, d, v) for v in (False, True)]
    values = np.zeros((2, rows, hkv, d))
    for s in range(len(kv)):
        for j in range(new[s]):
            row, p = row_start[s] + j, kv[s] - new[s] + j
            if rot:
                c, t = host(cs[p, :, 0]), host(cs[p, :, 1])
                a, b = x[row, hq:hq + hkv][:, first], x[row, hq:hq + hkv][:, second]
                keys[row][:, first], keys[row][:, second] = a * c - b * t, b * c + a * t
            for i, rows_of in enumerate((keys[row], x[row, hq + hkv:])):
                codes, scales = so.hold(rows_of)
                piece = want[i][table[s, p // page]]
                piece[:, at_bytes[i][0][p % page]] = codes[:, 0::2] | codes[:, 1::2] << 4
                piece[:, at_bytes[i][1][p % page]] = scales
                values[i, row] = so.held(codes, scales)
    for i, pool in enumerate((K, V)):
        assert np.array_equal(pool.cpu().numpy(), want[i]), i
    if hq:
        plain = [torch.zeros((n_pages, hkv, page, d), dtype=dtype, device="cuda") for _ in range(2)]
        Q2 = torch.empty((rows, hq * d), dtype=dtype, device="cuda")
        g.gelo_rope_append(ctx, QKV, hq, g.KvCache(*plain), batch, Q=Q2, table=cs, rot_dim=rot, layout=layout)
        assert torch.equal(Q, Q2) and torch.all(Q_all[:, hq * d:] == 7)
        before = QKV.clone()                                 # in place: the queries turn where they lie
        Kp, Vp = pools(n_pages, hkv, page, d, order=order)
        g.gelo_rope_append_fp4(ctx, QKV, hq, g.KvCacheFp4(Kp, Vp, page, d), batch, Q=QKV[:, :hq * d], table=cs, rot_dim=rot, layout=layout)
        assert torch.equal(QKV[:, :hq * d], Q) and torch.equal(QKV[:, hq * d:], before[:, hq * d:])
        assert torch.equal(Kp, K) and torch.equal(Vp, V)
    for out in (BF16, F32):
        (gotK, allK), (gotV, allV) = (padded(rows, hkv * d, hkv * d + 16, out) for _ in range(2))
        g.gelo_cache_rows_fp4(ctx, cache, batch, gotK, gotV)
        assert np.array_equal(host(gotK).reshape(values[0].shape), values[0]) and np.array_equal(host(gotV).reshape(values[1].shape), values[1])
        assert torch.all(allK[:, hkv * d:] == 7) and torch.all(allV[:, hkv * d:] == 7)
        alone = torch.empty_like(gotV)
        g.gelo_cache_rows_fp4(ctx, cache, batch, V=alone)
        assert torch.equal(alone, gotV)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_blocks_at_the_edges_of_the_format(ctx, dtype):
    """Ties, the scale's border on both sides, zeros of either sign, values below and beyond the scales, NaN and infinities; neighbouring blocks do not notice."""
    d, page = 128, 16
    x = torch.zeros((16, d), dtype=torch.float64)
    x[0, :9] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25])
    x[0, 32:41] = -x[0, :9] / 1024
    x[1, 0], x[1, 33], x[1, 64] = 7.0, 7.03125, 3.484375      # (one step of bfloat16 to either side)
    x[2] = -0.0
    x[3] = 2.0 ** -113
    x[3, 5] = 7 * 2.0 ** -110
    x[4] = 2.0 ** -120
    x[5] = 3.3e38
    x[5, 3] = -2.0 ** 127
    x[6, 40], x[7, 70], x[8, 127] = math.nan, math.inf, -math.inf
    x[6, 0] = x[7, 0] = x[8, 0] = 1.0
    x[9:] = torch.randn((7, d), generator=torch.Generator().manual_seed(3), dtype=torch.float64) * 10.0 ** torch.arange(-30, 40, 10)[:, None]
    x = x.to(dtype)
    K, V = pools(2, 1, page, d)
    batch = g.SeqBatch(torch.tensor([16], dtype=torch.int32).cuda(), torch.tensor([[1]], dtype=torch.int32).cuda(), 16,
                       row_start=torch.tensor([0, 16], dtype=torch.int32).cuda(), max_rows=16)
    QKV = torch.cat((x, x), 1).cuda()
    for rot in (0, 128):                                      # turned by nothing: cosine 1 and sine 0
        table = torch.zeros((16, rot // 2, 2), device="cuda") if rot else None
        if rot:
            table[..., 0] = 1
        cache = g.KvCacheFp4(K, V, page, d)
        g.gelo_rope_append_fp4(ctx, QKV, 0, cache, batch, table=table, rot_dim=rot)
        codes, scales = so.hold(host(x))
        if rot:                                               # 0 times NaN or infinity reaches the partner's block as well
            bad = ~torch.isfinite(x)
            both = (bad | bad.roll(64, 1)).view(16, 4, 32).any(-1).numpy()
            codes, scales = codes.copy(), np.where(both, 255, scales).astype(np.uint8)
            codes.reshape(16, 4, 32)[both] = 0
            zero = host(x) == 0                               # (-0 + 0 is 0)
            got, want = so.unpack(K.cpu().numpy(), page, d, False)[1, 0], so.held(codes, scales)
            assert np.array_equal(got, want, equal_nan=True) and zero.any()
        else:
            assert np.array_equal(K[1, 0].cpu().numpy(), so.pack(codes[None, None], scales[None, None], False)[0, 0])
        codes, scales = so.hold(host(x))
        assert np.array_equal(V[1, 0].cpu().numpy(), so.pack(codes[None, None], scales[None, None], True)[0, 0])
        assert torch.all(K[0] == 0xA5) and torch.all(V[0] == 0xA5)
        back = torch.empty((16, d), dtype=dtype, device="cuda")
        g.gelo_cache_rows_fp4(ctx, cache, batch, V=back)
        assert np.array_equal(host(back), so.held(codes, scales), equal_nan=True)


def test_a_turned_key_beyond_float(ctx):
    """a cos - b sin of two of bfloat16's largest values is 4.7e38: the largest level, not NaN."""
    d, page = 64, 16
    K, V = pools(1, 1, page, d)
    QKV = torch.zeros((1, 2 * d), dtype=BF16, device="cuda")
    QKV[0, 3], QKV[0, 35] = 3.3e38, -3.3e38
    table = torch.full((1, 32, 2), math.sqrt(0.5), device="cuda")
    batch = g.SeqBatch(torch.ones(1, dtype=torch.int32).cuda(), torch.zeros((1, 1), dtype=torch.int32).cuda(), 1)
    g.gelo_rope_append_fp4(ctx, QKV, 0, g.KvCacheFp4(K, V, page, d), batch, table=table, rot_dim=d)
    got = so.unpack(K.cpu().numpy(), page, d, False)[0, 0, 0]
    assert got[3] == 6 * 2.0 ** 125 and got[35] == 0


def test_rows_that_have_no_place(ctx):
    """A position below zero, one at the bound, a page number outside the cache, a row of no sequence."""
    page, d = 16, 64
    K, V = pools(4, 1, page, d)
    table = torch.tensor([[0, 1], [2, 3], [4, -1], [-7, 0]], dtype=torch.int32, device="cuda")
    kv = torch.tensor([1, 33, 5, 7], dtype=torch.int32, device="cuda")
    row_start = torch.tensor([0, 2, 4, 5, 6], dtype=torch.int32, device="cuda")
    batch = g.SeqBatch(kv, table, 32, row_start=row_start, max_rows=2)
    QKV = rand((8, 3 * d), 3, BF16)
    Q = torch.full((8, d), 7.0, dtype=BF16, device="cuda")
    cache = g.KvCacheFp4(K, V, page, d)
    g.gelo_rope_append_fp4(ctx, QKV, 1, cache, batch, Q=Q)
    assert torch.all(Q[0] == 0) and torch.isnan(Q[3]).all() and torch.all(Q[6:] == 7)
    for r in (1, 2, 4, 5):
        assert torch.equal(Q[r], QKV[r, :d])
    for pool, values in ((K, False), (V, True)):
        at, at_scale = so.places(page, d, values)
        touched = np.zeros(pool.shape, dtype=bool)
        for p, r in ((0, 0), (3, 15)):
            touched[p, 0, at[r]] = touched[p, 0, at_scale[r]] = True
        assert np.all(pool.cpu().numpy()[~touched] == 0xA5)
    k, v = (torch.full((8, d), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    g.gelo_cache_rows_fp4(ctx, cache, batch, k, v)
    for got, first in ((k, d), (v, 2 * d)):
        assert torch.all(got[0] == 0) and torch.isnan(got[3:6]).all() and torch.all(got[6:] == 7)
        want = so.held(*so.hold(host(QKV[:, first:first + d])))
        assert np.array_equal(host(got[1:3]), want[1:3])


# ----------------------------------------------------------------------------------------------------- attention --
def attention_bound(ref, absolute, Q, K, scale, kv, d, dtype):
    """As for the attention over values: a score is a sum of d products, scaled, (d + 6) U32 of |q| |k| scale, which the exponential makes a relative error
    of its weight; the sums over the keys err by a U32 per key and rescaling; all of it twice (weights and their sum) on sum w |v|.  A float query or
    weight is three bfloat16, so three products and sums to each.  bfloat16: a weight rounded, in its sum too, which is U16 of sum w |v| + |O| at
    most; the result rounded once."""
    parts = 3 if dtype == F32 else 2
    q = np.linalg.norm(Q.reshape(-1, d), axis=1).max()
    k = np.linalg.norm(np.nan_to_num(K, nan=0.0).reshape(-1, d), axis=1).max()
    e = U32 * parts * ((d + 6) * abs(scale) * q * k + kv + 64)
    bound = 2 * e * absolute
    if dtype == BF16:
        bound = bound + 1.01 * U16 * (absolute + 2 * np.abs(ref))
    return bound + 1e-30


def hide(K, V, table, kv, page, d, byte=255):
    """Everything that no query may see - rows behind a sequence's end, pages of nobody - becomes such bytes; 255: NaN."""
    n_pages = K.shape[0]
    seen = np.zeros((n_pages, page), dtype=bool)
    for s, n in enumerate(kv):
        for p in range(n):
            seen[table[s, p // page], p % page] = True
    for pool, values in ((K, False), (V, True)):
        at, at_scale = so.places(page, d, values)
        mask = np.ones((n_pages, so.piece_bytes(page, d)), dtype=bool)
        for places in (at, at_scale):
            for r in range(page):
                mask[np.ix_(seen[:, r], places[r])] = False
        pool.masked_fill_(torch.from_numpy(mask).cuda()[:, None], byte)


def run_attention(ctx, dtype, new, kv, hq, hkv, d, page, order, causal, scale=None, max_kv=None, one_row=False, seed=7, heads=None):
    batch, table, row_start, n_pages = make_batch(new, kv, page, seed, max_kv=max_kv, one_row=one_row)
    rows = int(row_start[-1])
    K, V, k, v = filled(n_pages, hkv, page, d, seed, order)
    hide(K, V, table, kv, page, d)
    Q, _ = padded(rows, hq * d, hq * d + 40, dtype)
    Q.copy_(rand(Q.shape, seed + 3, dtype))
    O, O_all = padded(rows, hq * d, hq * d + 16, dtype)
    scale = 1 / math.sqrt(d) if scale is None else scale
    g.gelo_attention_fp4(ctx, Q, O, hq, g.KvCacheFp4(K, V, page, d), batch, scale, causal=causal)
    assert torch.all(O_all[:, hq * d:] == 7)
    for h in range(hq) if heads is None else heads:
        kh = h * hkv // hq
        at = slice(h * d, (h + 1) * d)
        ref, absolute = lo.attention(host(Q[:, at]), k[:, kh:kh + 1], v[:, kh:kh + 1], 1, row_start, kv, table, scale, causal)
        within(O[:, at], ref, attention_bound(ref, absolute, host(Q[:, at]), k[:, kh], scale, max(kv), d, dtype), h)
    return O


DECODES = [  # kv, q heads, kv heads, d, page, order
    ([1], 1, 1, 64, 16, "pages"),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33], 4, 4, 128, 16, "pages"),
    ([127, 128, 129, 255, 256, 257, 0], 6, 2, 64, 64, "heads"),
    ([300, 5], 14, 2, 96, 32, "both"),
    ([77, 1030], 16, 1, 256, 16, "pages"),
    ([513, 40], 48, 2, 64, 128, "both"),
    ([2100], 8, 8, 128, 64, "heads"),
    ([63, 64, 65, 47, 48, 49], 3, 3, 96, 16, "pages"),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kv,hq,hkv,d,page,order", DECODES)
def test_attention_of_single_tokens(ctx, dtype, kv, hq, hkv, d, page, order):
    run_attention(ctx, dtype, [1] * len(kv), kv, hq, hkv, d, page, order, True, one_row=True)


def way(dtype, new, kv, hq, hkv, d, causal=True):
    """0: few columns to a key head, 1: many, 2: many in pairs; plus 4 where the cache is cut, 8 where a wave has a head to itself."""
    return ctypes.CDLL(g.LIB_PATH)["_ZN4gelo17attention_fp4_wayEiiiiiiiii"](int(dtype == BF16), int(causal), hq, hkv, d, len(kv), sum(new), max(new), max(kv))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kv,hq,hkv,d,chunks", [([16500, 300, 0, 4224, 4225, 8449, 1] + [17] * 123, 4, 2, 64, 4), ([20481, 5, 9000], 64, 64, 96, 5)])
def test_long_caches_are_cut_beyond_what_fills_the_chip(ctx, kv, hq, hkv, d, chunks, dtype):
    """Sequences that end in the first piece, at a piece's end, in none."""
    parts = ctypes.CDLL(g.LIB_PATH)["_ZN4gelo19attention_fp4_partsEiiiiiiiii"]
    parts.restype = ctypes.c_size_t
    n = len(kv)
    assert parts(int(dtype == BF16), 1, hq, hkv, d, n, n, 1, max(kv)) == chunks * n * hq * (d + 2) * 4
    run_attention(ctx, dtype, [1] * n, kv, hq, hkv, d, 64, "pages", True, one_row=True, heads=(0, hq - 1))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,hq,order", [(64, 16, "pages"), (96, 32, "heads"), (128, 16, "both"), (256, 48, "pages")])
def test_single_tokens_of_many_sequences(ctx, dtype, d, hq, order):
    """So many sequences and heads that a wave has a head of its own; lengths at the edges of tiles and steps."""
    kv = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 129] * 11
    assert way(dtype, [1] * len(kv), kv, hq, 16, d) == (0 if dtype == F32 and d >= 128 else 8)
    run_attention(ctx, dtype, [1] * len(kv), kv, hq, 16, d, 16, order, True, one_row=True, seed=2, heads=(0, hq // 2 + 1, hq - 1))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_where_the_bound_is_far_above_the_lengths(ctx, dtype):
    """A captured launch is sized for the longest context: chunks that no sequence reaches."""
    run_attention(ctx, dtype, [1] * 3, [3, 700, 0], 4, 2, 128, 16, "pages", True, one_row=True, max_kv=9000)


PROMPTS = [  # new rows, kv, q heads, kv heads, d, page, order, causal
    ([1, 5], [1, 5], 2, 2, 64, 16, "pages", True),
    ([16, 17, 0, 33], [16, 17, 4, 33], 4, 1, 128, 16, "heads", True),
    ([64, 65], [64, 200], 2, 2, 128, 64, "pages", True),
    ([3, 20], [2, 7], 3, 3, 64, 32, "both", True),               # more new rows than the cache holds: the first ones see nothing
    ([129], [129], 3, 1, 96, 16, "pages", True),
    ([130, 40], [700, 41], 4, 2, 64, 32, "heads", True),
    ([31, 70], [33, 71], 2, 1, 256, 16, "pages", True),
    ([257], [300], 5, 5, 128, 128, "both", True),
    ([2], [1500], 8, 1, 128, 16, "pages", True),
    ([5, 33, 12], [1, 100, 0], 4, 4, 64, 16, "pages", False),     # cross attention, one sequence without states
    ([70, 200], [257, 64], 2, 2, 128, 64, "heads", False),
    ([9], [130], 12, 2, 96, 32, "pages", False),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new,kv,hq,hkv,d,page,order,causal", PROMPTS)
def test_attention_of_prompts(ctx, dtype, new, kv, hq, hkv, d, page, order, causal):
    run_attention(ctx, dtype, new, kv, hq, hkv, d, page, order, causal)


LARGE = [  # dtype, new rows, kv, q heads, kv heads, d, page, order, causal
    (BF16, [512, 377, 512, 1, 130, 512, 256, 400], [512, 377, 600, 1, 130, 512, 256, 400], 32, 32, 128, 16, "pages", True),
    (BF16, [384, 200, 384, 384, 129, 384, 300, 384], [384, 200, 384, 500, 129, 384, 300, 384], 32, 32, 128, 64, "heads", True),
    (BF16, [384, 130, 384, 70], [384, 130, 390, 70], 32, 32, 256, 32, "pages", True),
    (BF16, [390, 128] * 4, [390, 300] * 4, 32, 32, 64, 16, "both", True),
    (BF16, [200], [5000], 8, 8, 64, 64, "pages", True),
    (BF16, [65, 200], [3000, 4111], 12, 4, 96, 16, "heads", False),
    (BF16, [90], [7000], 16, 4, 128, 32, "pages", True),
    (BF16, [300, 20], [2500, 90], 8, 4, 256, 16, "pages", True),
    (BF16, [1500], [2777], 14, 2, 128, 128, "pages", True),
    (BF16, [1, 1], [30011, 9], 16, 2, 128, 64, "pages", True),
    (F32, [1], [20000], 8, 2, 96, 16, "heads", True),
    (F32, [700, 33], [1300, 33], 8, 2, 128, 64, "pages", True),
    (F32, [40, 33], [1300, 33], 8, 2, 256, 64, "pages", True),
    (BF16, [1, 1, 1], [4100, 3000, 1], 48, 2, 64, 32, "pages", True),
]


@pytest.mark.parametrize("dtype,new,kv,hq,hkv,d,page,order,causal", LARGE)
def test_attention_at_the_sizes_where_launches_differ(ctx, dtype, new, kv, hq, hkv, d, page, order, causal):
    """The reference in float64 on the GPU, for every sequence and two of the heads; the same bound as above."""
    batch, table, row_start, n_pages = make_batch(new, kv, page, 3, one_row=max(new) == 1)
    rows = int(row_start[-1])
    K, V = pools(n_pages, hkv, page, d, order=order)
    rng = np.random.default_rng(5)
    codes = [rng.integers(0, 16, (n_pages, hkv, page, d), dtype=np.uint8) for _ in range(2)]
    scales = [rng.integers(124, 127, (n_pages, hkv, page, d // 32), dtype=np.uint8) for _ in range(2)]
    for pool, c, s, values in zip((K, V), codes, scales, (False, True)):
        pool.copy_(torch.from_numpy(so.pack(c, s, values)))
    held = [torch.from_numpy(so.held(c, s)) for c, s in zip(codes, scales)]
    Q, O = rand((rows, hq * d), 8, dtype), torch.full((rows, hq * d), 7.0, dtype=dtype, device="cuda")
    g.gelo_attention_fp4(ctx, Q, O, hq, g.KvCacheFp4(K, V, page, d), batch, 1 / math.sqrt(d), causal=causal)
    assert torch.isfinite(O.float()).all()
    for s in range(len(kv)):
        used = torch.from_numpy(table[s, :(kv[s] + page - 1) // page]).long()
        at = slice(int(row_start[s]), int(row_start[s + 1]))
        for h in {0, (7 * s + 5) % hq}:
            kh = h * hkv // hq
            k, v = (x[used, kh].reshape(-1, d)[:kv[s]].cuda() for x in held)
            q = Q[at, h * d:(h + 1) * d].double()
            score = q @ k.T / math.sqrt(d)
            if causal:
                score.masked_fill_(torch.arange(kv[s], device="cuda")[None] > torch.arange(new[s], device="cuda")[:, None] + (kv[s] - new[s]), -math.inf)
            w = torch.softmax(score, -1)
            ref, absolute = host(w @ v), host(w @ v.abs())
            within(O[at, h * d:(h + 1) * d], ref, attention_bound(ref, absolute, host(q), host(k), 1 / math.sqrt(d), kv[s], d, dtype), (s, h))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
@pytest.mark.parametrize("new,kv,hq", [([1, 20], [90, 150], 4), ([150] * 16, [150 + 9 * i for i in range(16)], 16)])
def test_attention_scales(ctx, dtype, new, kv, hq, scale):
    """Equal weights, reversed ones, and scores so far apart that a single key is left."""
    run_attention(ctx, dtype, new, kv, hq, hq // 2, 64, 16, "pages", True, scale=scale, heads=(0, hq - 1))


EDGES = [(1, 1), (5, 1), (16, 16), (17, 17), (31, 40), (32, 32), (33, 63), (63, 64), (64, 65), (65, 64), (127, 128), (128, 127), (129, 200), (2, 0), (0, 9),
         (140, 15), (64, 191), (96, 192), (130, 193), (20, 257), (257, 300), (48, 48), (200, 112), (70, 129)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,hq,hkv,page,order", [(64, 32, 16, 16, "pages"), (96, 16, 16, 32, "heads"), (128, 32, 16, 16, "both"), (256, 16, 16, 64, "pages")])
def test_many_columns_at_the_edges_of_tiles(ctx, d, hq, hkv, page, order, causal):
    """The kernel for prompts.  New rows and lengths at, before and behind the ends of tiles, steps and groups, none, and more rows than keys; rows of the cache that
    belong to nobody are NaN.  All rows of three heads."""
    assert way(BF16, [x[0] for x in EDGES], [x[1] for x in EDGES], hq, hkv, d, causal) in (1, 2)
    run_attention(ctx, BF16, [x[0] for x in EDGES], [x[1] for x in EDGES], hq, hkv, d, page, order, causal, seed=3, heads=(0, hq // 2 + 1, hq - 1))


ODD = [  # dtype, sequences, rows, heads, page, the ways it goes at the widths in turn
    (BF16, 2, 1, 4, 16, (0, 0, 0, 0)), (F32, 2, 1, 4, 16, (0, 0, 0, 0)), (BF16, 1, 12, 1, 16, (0, 0, 0, 0)), (F32, 1, 150, 2, 32, (0, 0, 0, 0)),
    (BF16, 16, 150, 16, 16, (1, 1, 1, 2)), (BF16, 8, 512, 16, 16, (1, 1, 1, 2)), (BF16, 16, 384, 16, 16, (2, 2, 2, 1)), (BF16, 132, 1, 16, 16, (8, 8, 8, 8))]


@pytest.mark.parametrize("dtype,n_seqs,rows,heads,page,ways", ODD)
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_blocks_that_are_nan_reach_only_rows_that_see_them(ctx, d, dtype, n_seqs, rows, heads, page, ways):
    """One block of one value row in every sequence and head: only query rows from its own on, and only that block's components; everything else keeps its bits.  A
    key's block: the rows before it do not see it.  A page number outside the cache: its sequence alone."""
    kv = max(rows, 90)
    at, block = 75, 1
    assert way(dtype, [rows] * n_seqs, [kv] * n_seqs, heads, heads, d) == ways[(64, 96, 128, 256).index(d)]
    each = (kv + page - 1) // page
    K, V, _, _ = filled(n_seqs * each, heads, page, d, 3)
    table = torch.arange(n_seqs * each, dtype=torch.int32, device="cuda").view(n_seqs, each)
    row_start = (torch.arange(n_seqs + 1, device="cuda") * rows).int()
    batch = g.SeqBatch(torch.full((n_seqs,), kv, dtype=torch.int32).cuda(), table, kv, row_start=row_start, max_rows=rows)
    pages = table[:, at // page].long()
    Q = rand((n_seqs * rows, heads * d), 9, dtype)

    def run(k, v, b=batch):
        O = torch.empty_like(Q)
        g.gelo_attention_fp4(ctx, Q, O, heads, g.KvCacheFp4(k, v, page, d), b, 1 / math.sqrt(d))
        return O.view(n_seqs, rows, heads, d)
    clean = run(K, V)
    assert torch.isfinite(clean.float()).all()
    first = max(at - (kv - rows), 0)                         # the first query row that sees it
    odd = V.clone()
    odd[pages, :, so.scale_byte(page, d, at % page, block, True)] = 255
    # without it, for the other blocks: its scale stands for what the kernels may put in its place
    o = run(K, odd)
    mine = torch.arange(d, device="cuda") // 32 == block
    assert torch.equal(o[..., ~mine], clean[..., ~mine]) and torch.equal(o[:, :first], clean[:, :first])
    assert torch.isnan(o[:, first:][..., mine]).all()
    odd = K.clone()
    odd[pages, :, so.scale_byte(page, d, at % page, block, False)] = 255
    o = run(odd, V)
    assert torch.equal(o[:, :first], clean[:, :first]) and torch.isnan(o[:, first:]).all()
    bad = table.clone()
    bad[n_seqs - 1, 2] = n_seqs * each
    o = run(K, V, g.SeqBatch(batch.kv_len, bad, kv, row_start=row_start, max_rows=rows))
    assert torch.equal(o[:-1], clean[:-1]) and torch.isnan(o[-1, -1]).all()
    bad[n_seqs - 1, 2] = -3
    assert torch.isnan(run(K, V, g.SeqBatch(batch.kv_len, bad, kv, row_start=row_start, max_rows=rows))[-1, -1]).all()


@pytest.mark.parametrize("dtype,new,kv,heads", [(BF16, [1, 1, 1], [1, 77, 2050], 2), (F32, [3, 40], [3, 75], 2), (BF16, [1] * 132, [70] * 132, 16), (BF16, [150] * 16, [155] * 16, 16)])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_nothing_that_lies_where_nobody_sees_it_is_felt(ctx, d, dtype, new, kv, heads):
    """Rows behind a sequence's end that were never written may hold any byte, scales that no append writes among them: with 253 and 254 there the values are infinite."""
    batch, table, row_start, n_pages = make_batch(new, kv, 16, 6)
    K, V, _, _ = filled(n_pages, heads, 16, d, 5)
    Q = rand((int(row_start[-1]), heads * d), 8, dtype)
    results = []
    for byte in (0, 127, 252, 253, 254, 255):
        hide(K, V, table, kv, 16, d, byte)
        results.append(torch.empty_like(Q))
        g.gelo_attention_fp4(ctx, Q, results[-1], heads, g.KvCacheFp4(K, V, 16, d), batch, d ** -0.5)
        assert torch.isfinite(results[-1].float()).all(), byte
        assert torch.equal(results[-1], results[0]), byte


@pytest.mark.parametrize("dtype,new,hq", [(BF16, [1] * 5, 4), (F32, [1] * 5, 4), (BF16, [150] * 8, 16), (F32, [40] * 3, 2)])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_a_row_that_sees_one_key_is_its_value(ctx, new, hq, dtype, d):
    """Weight times value over weight: the value up to the quotient's two roundings (and the sum's parts): 8 U32, which bfloat16 rounds away, since values that
    are held are two bits."""
    batch, table, row_start, n_pages = make_batch(new, [1] * len(new), 16, 3)
    K, V, _, v = filled(n_pages, hq, 16, d, 5)
    Q = rand((int(row_start[-1]), hq * d), 8, dtype)
    O = torch.full_like(Q, 7.0)
    g.gelo_attention_fp4(ctx, Q, O, hq, g.KvCacheFp4(K, V, 16, d), batch, 1 / math.sqrt(d), causal=False)
    for s in range(len(new)):
        want = np.broadcast_to(v[table[s, 0], :, 0], (new[s], hq, d))
        within(O[int(row_start[s]):int(row_start[s + 1])].view(-1, hq, d), want, (0.0 if dtype == BF16 else 8 * U32) * np.abs(want))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_queries_and_scores_at_the_ends_of_float(ctx, dtype):
    """Large finite scores leave one key; an infinity in a query makes its row's head NaN and no other."""
    n, hq, d = 40, 2, 64
    batch, table, row_start, n_pages = make_batch([n], [n + 30], 16, 3)
    K, V, k, v = filled(n_pages, hq, 16, d, 5)
    Q = rand((n, hq * d), 8, dtype)
    O, far = torch.empty_like(Q), torch.empty_like(Q)
    cache = g.KvCacheFp4(K, V, 16, d)
    g.gelo_attention_fp4(ctx, Q, O, hq, cache, batch, 0.125)
    odd = Q.clone()
    odd[7, 5] = math.inf
    odd[9, d + 3] = math.nan
    odd[11, :d] *= 1e30
    g.gelo_attention_fp4(ctx, odd, far, hq, cache, batch, 0.125)
    o, f = O.view(n, hq, d), far.view(n, hq, d)
    assert torch.isnan(f[7, 0]).all() and torch.isnan(f[9, 1]).all()
    same = torch.ones((n, hq), dtype=torch.bool)
    same[7, 0] = same[9, 1] = same[11, 0] = False
    assert torch.equal(o[same], f[same])
    keys = lo.cache_rows(k, table[0], 0, n + 30)[:30 + 12]
    values = lo.cache_rows(v, table[0], 0, n + 30)[:30 + 12]
    score = keys @ host(Q[11, :d])
    assert np.sort(score)[-1] - np.sort(score)[-2] > 1e-3
    within(f[11, 0], values[score.argmax()], 8 * U32 * np.abs(values[score.argmax()]))


@pytest.mark.parametrize("new", [1, 70])
def test_a_cache_beyond_32_bit_offsets(ctx, new):
    """Pages whose bytes lie behind 2^31: 70000 pages of 16 rows of 16 heads of 256 values are 2.4e9 bytes each."""
    heads, d, page, n_pages = 16, 256, 16, 70000
    piece = so.piece_bytes(page, d)
    K, V = (torch.zeros((n_pages, heads, piece), dtype=torch.uint8, device="cuda") for _ in range(2))
    kv = 90
    pages = torch.tensor([[n_pages - 1 - 3 * i for i in range(6)]], dtype=torch.int32, device="cuda")
    batch = g.SeqBatch(torch.tensor([kv], dtype=torch.int32).cuda(), pages, kv, row_start=torch.tensor([0, new], dtype=torch.int32).cuda(), max_rows=new)
    fill = g.SeqBatch(torch.tensor([kv], dtype=torch.int32).cuda(), pages, kv, row_start=torch.tensor([0, kv], dtype=torch.int32).cuda(), max_rows=kv)
    QKV = rand((kv, 3 * heads * d), 5, BF16)
    cache = g.KvCacheFp4(K, V, page, d)
    whole = torch.empty((kv, heads * d), dtype=BF16, device="cuda")
    g.gelo_rope_append_fp4(ctx, QKV, heads, cache, fill, Q=whole)
    small = [torch.zeros((6, heads, piece), dtype=torch.uint8, device="cuda") for _ in range(2)]
    near = torch.arange(6, dtype=torch.int32, device="cuda")[None]
    small_cache, near_fill = g.KvCacheFp4(*small, page, d), g.SeqBatch(fill.kv_len, near, kv, row_start=fill.row_start, max_rows=kv)
    g.gelo_rope_append_fp4(ctx, QKV, heads, small_cache, near_fill, Q=whole)
    assert torch.equal(K[pages[0].long()], small[0]) and torch.equal(V[pages[0].long()], small[1])
    rows = [torch.empty((kv, heads * d), dtype=BF16, device="cuda") for _ in range(4)]
    g.gelo_cache_rows_fp4(ctx, cache, fill, *rows[:2])
    g.gelo_cache_rows_fp4(ctx, small_cache, near_fill, *rows[2:])
    assert torch.equal(rows[0], rows[2]) and torch.equal(rows[1], rows[3])
    Q = whole[kv - new:].contiguous()
    O, want = torch.empty_like(Q), torch.empty_like(Q)
    g.gelo_attention_fp4(ctx, Q, O, heads, cache, batch, 1 / 16)
    g.gelo_attention_fp4(ctx, Q, want, heads, small_cache, g.SeqBatch(batch.kv_len, near, kv, row_start=batch.row_start, max_rows=new), 1 / 16)
    assert torch.equal(O, want) and O.float().abs().sum() > 0


def test_rows_of_no_sequence_are_left_alone(ctx):
    K, V, _, _ = filled(8, 1, 16, 64, 3)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    row_start = torch.tensor([2, 5, 7], dtype=torch.int32).cuda()
    for max_kv in (64, 40):
        batch = g.SeqBatch(torch.tensor([40, 9], dtype=torch.int32).cuda(), table, max_kv, row_start=row_start, max_rows=3)
        Q = rand((10, 64), 9, BF16)
        O = torch.full_like(Q, 7.0)
        g.gelo_attention_fp4(ctx, Q, O, 1, g.KvCacheFp4(K, V, 16, 64), batch, 0.125)
        assert torch.all(O[:2] == 7) and torch.all(O[7:] == 7) and torch.all(O[2:7] != 7)


@pytest.mark.parametrize("which", ["kv_len", "row_start"])
@pytest.mark.parametrize("value", [-2 ** 31, -1, 2 ** 31 - 1])
def test_lengths_and_row_starts_at_the_ends_of_32_bits(ctx, which, value):
    """What the host cannot see is bounded in the kernels: the other sequence keeps its bits, nothing outside the cache is read or written."""
    page, d, heads = 16, 64, 2
    K, V, _, _ = filled(8, heads, page, d, 3)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    kv = torch.tensor([40, 40], dtype=torch.int32).cuda()
    start = torch.tensor([0, 20, 40], dtype=torch.int32).cuda()
    Q = rand((40, heads * d), 9, BF16)
    want, O = torch.empty_like(Q), torch.empty_like(Q)
    g.gelo_attention_fp4(ctx, Q, want, heads, g.KvCacheFp4(K, V, page, d), g.SeqBatch(kv, table, 64, row_start=start, max_rows=20), 0.125)
    (kv if which == "kv_len" else start)[-1] = value
    batch = g.SeqBatch(kv, table, 64, row_start=start, max_rows=20)
    g.gelo_attention_fp4(ctx, Q, O, heads, g.KvCacheFp4(K, V, page, d), batch, 0.125)
    assert torch.equal(O[:20], want[:20])
    before = K.clone()
    QKV = rand((40, 3 * heads * d), 4, BF16)
    g.gelo_rope_append_fp4(ctx, QKV, heads, g.KvCacheFp4(K, V, page, d), batch, Q=O)
    g.gelo_cache_rows_fp4(ctx, g.KvCacheFp4(K, V, page, d), batch, want)
    if which == "kv_len":                                    # (row starts that do not ascend say nothing about other rows)
        assert torch.equal(K[0], before[0]) and not torch.equal(K[1], before[1])          # rows 20 ... 39 of the first sequence
        assert torch.isfinite(want[:20].float()).all()


def serve(ctx, s):
    """The run of calls of a decode step with adapters: projection's addition, append, attention."""
    g.gelo_adapt(ctx, s["H"], s["adapters"], s["which"], s["QKV"], base=s["Z"])
    g.gelo_rope_append_fp4(ctx, s["QKV"], 4, s["cache"], s["batch"], Q=s["Q"], table=s["table"], rot_dim=64)
    g.gelo_attention_fp4(ctx, s["Q"], s["O"], 4, s["cache"], s["batch"], 0.125)


def serve_state(ctx, kv, seed):
    batch, _, _, n_pages = make_batch([1] * len(kv), kv, 16, seed, max_kv=3000, one_row=True)
    K, V, _, _ = filled(n_pages, 2, 16, 64, seed)
    n = len(kv)
    empty = lambda w: torch.empty((n, w), dtype=BF16, device="cuda")  # noqa: E731
    return {"H": rand((n, 256), seed, BF16), "Z": rand((n, 512), seed + 1, BF16), "QKV": empty(512), "Q": empty(256), "O": empty(256),
            "adapters": g.Adapters(rand((3, 24, 256), seed + 2, BF16, 0.06), rand((3, 512, 8), seed + 3, BF16), part_ends=[256, 384, 512]),
            "which": torch.tensor([i % 4 - 1 for i in range(n)], dtype=torch.int32).cuda(), "cache": g.KvCacheFp4(K, V, 16, 64), "batch": batch,
            "table": g.gelo_rope_table(ctx, 64, 3000)}


def test_other_streams_and_captured_graphs(ctx):
    """The calls on a stream of their own, and captured once and replayed for other inputs in the same buffers, against plain calls."""
    g.gelo_reserve_attention(ctx, 64)
    g.gelo_reserve_adapt(ctx, 4, 8, 3, 3)
    a = serve_state(ctx, [2500, 40, 7, 0], 20)
    pool = a["cache"].K.clone(), a["cache"].V.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        serve(ctx, a)
    side.synchronize()
    O_side, K_side = a["O"].clone(), a["cache"].K.clone()
    a["cache"].K.copy_(pool[0]), a["cache"].V.copy_(pool[1]), a["O"].fill_(3)
    serve(ctx, a)
    torch.cuda.synchronize()
    assert torch.equal(a["O"], O_side) and torch.equal(a["cache"].K, K_side)
    assert torch.all(a["O"][3] == 0)                                   # kv_len 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        serve(ctx, a)
    for turn, lens in enumerate(([2500, 40, 7, 0], [2501, 41, 8, 1], [3, 2600, 0, 100], [1, 1, 1, 1])):
        for key, width in (("H", 256), ("Z", 512)):
            a[key].copy_(rand((4, width), 50 + turn, BF16))
        a["which"].copy_(torch.tensor([turn, 2, -1, turn - 1], dtype=torch.int32))
        a["batch"].page_table.copy_(torch.arange(4 * 188, dtype=torch.int32).view(4, 188) % a["cache"].K.shape[0])
        a["batch"].kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        a["cache"].K.copy_(pool[0]), a["cache"].V.copy_(pool[1])
        graph.replay()
        torch.cuda.synchronize()
        got = [a[x].clone() for x in ("QKV", "Q", "O")] + [a["cache"].K.clone(), a["cache"].V.clone()]
        a["cache"].K.copy_(pool[0]), a["cache"].V.copy_(pool[1])
        serve(ctx, a)
        torch.cuda.synchronize()
        for x, y in zip([a[x] for x in ("QKV", "Q", "O")] + [a["cache"].K, a["cache"].V], got):
            assert torch.equal(x, y)


@pytest.mark.parametrize("later", ["fp4", "plain"])
def test_workspace_that_is_outgrown_serves_captured_calls(ctx, later):
    """A captured call keeps its workspace's address: a call later that needs more, of either kind of cache, takes another one."""
    c = g.gelo_create(0, 1)
    try:
        a, b = ([1], [2500], 2, 64), ([1] * 4, [4000] * 4, 4, 256)
        lib = ctypes.CDLL(g.LIB_PATH)

        def needs(new, kv, heads, d):
            parts = getattr(lib, "_ZN4gelo19attention_fp4_partsEiiiiiiiii")
            parts.restype = ctypes.c_size_t
            return parts(1, 1, heads, heads, d, len(new), len(new), 1, max(kv))
        assert 0 < 2 * needs(*a) < needs(*b)

        def state(new, kv, heads, d):
            batch, _, _, n_pages = make_batch(new, kv, 16, 3, one_row=True)
            Q = rand((len(new), heads * d), 4, BF16)
            K, V, _, _ = filled(n_pages, heads, 16, d, 5)
            return Q, torch.empty_like(Q), heads, g.KvCacheFp4(K, V, 16, d), batch, d ** -0.5
        small, large = state(*a), state(*b)
        g.gelo_attention_fp4(c, *small)
        want = small[1].clone()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            g.gelo_attention_fp4(c, *small)
        if later == "fp4":
            g.gelo_attention_fp4(c, *large)
        else:
            pool = rand((4 * 250 + 3, 4, 16, 256), 6, BF16)
            g.gelo_attention(c, large[0], large[1], 4, g.KvCache(pool, pool), large[4], 0.1)
        hold = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(8)]        # what the runtime may put into memory that was given back
        for _ in range(3):
            small[1].fill_(5)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(small[1], want)
            if later == "fp4":
                g.gelo_attention_fp4(c, *large)
        del hold
    finally:
        g.gelo_destroy(c)


def test_the_same_call_twice_gives_the_same_bits(ctx):
    O = run_attention(ctx, BF16, [1, 1], [2000, 1111], 8, 2, 128, 16, "pages", True, one_row=True)
    assert torch.equal(O, run_attention(ctx, BF16, [1, 1], [2000, 1111], 8, 2, 128, 16, "pages", True, one_row=True))


def test_a_run_of_append_and_attention_token_by_token(ctx):
    """A prompt and then tokens, each appended before it attends, against the prompt and tokens in one call: the same held rows, results as near as their bounds."""
    heads, kvh, d, page, n = 6, 2, 128, 16, 45
    QKV = rand((n, (heads + 2 * kvh) * d), 5, BF16)
    cs = g.gelo_rope_table(ctx, d, n)
    table = torch.randperm(5, generator=torch.Generator().manual_seed(1)).int().cuda()[None]
    Q, O = (torch.empty((n, heads * d), dtype=BF16, device="cuda") for _ in range(2))
    one, many = (g.KvCacheFp4(*pools(5, kvh, page, d), page, d) for _ in range(2))
    whole = g.SeqBatch(torch.tensor([n], dtype=torch.int32).cuda(), table, n, row_start=torch.tensor([0, n], dtype=torch.int32).cuda(), max_rows=n)
    g.gelo_rope_append_fp4(ctx, QKV, heads, one, whole, Q=Q, table=cs, rot_dim=d)
    g.gelo_attention_fp4(ctx, Q, O, heads, one, whole, d ** -0.5)
    k, v = (so.unpack(x.cpu().numpy(), page, d, values) for x, values in ((one.K, False), (one.V, True)))
    got = torch.empty_like(O)
    for first, last in ((0, 30), *((i, i + 1) for i in range(30, n))):
        batch = g.SeqBatch(torch.tensor([last], dtype=torch.int32).cuda(), table, n, row_start=torch.tensor([0, last - first], dtype=torch.int32).cuda(), max_rows=last - first)
        q = torch.empty((last - first, heads * d), dtype=BF16, device="cuda")
        g.gelo_rope_append_fp4(ctx, QKV[first:last], heads, many, batch, Q=q, table=cs, rot_dim=d)
        g.gelo_attention_fp4(ctx, q, got[first:last], heads, many, batch, d ** -0.5)
    assert torch.equal(one.K, many.K) and torch.equal(one.V, many.V)
    ref, absolute = lo.attention(host(Q), k, v, heads, [0, n], [n], table.cpu().numpy(), d ** -0.5, True)
    bound = attention_bound(ref, absolute, host(Q), k[table.cpu().numpy()[0]][:3], d ** -0.5, n, d, BF16)
    within(O, ref, bound)
    within(got, ref, bound)


# ------------------------------------------------------------------------------------------------------ refusals --
def test_refusals(ctx):
    lib, P = g.load_library(), ctypes.c_void_p
    buf = torch.full((1 << 16,), 5.0, device="cuda")
    ints = torch.zeros(64, dtype=torch.int32, device="cuda")
    x, i = buf.data_ptr(), ints.data_ptr()
    piece = so.piece_bytes(16, 64)

    def structs(**kw):
        c = dict(k=x, v=x, n_pages=2, n_kv_heads=2, page_rows=16, head_dim=64, page_stride=2 * piece, head_stride=piece)
        b = dict(n_seqs=2, n_rows=2, max_rows=1, max_kv_len=32, row_start=None, kv_len=i, page_table=i, table_ld=2)
        for k, v in kw.items():
            (c if k in c else b)[k] = v
        return g._KvCacheFp4Struct(*c.values()), g._SeqBatchStruct(*b.values())

    def append(dtype=0, hq=4, ld=512, layout=0, rot=64, table=x, n_table=32, Q=x, ldq=256, **kw):
        c, b = structs(**kw)
        return g.STATUS_NAMES[lib.gelo_rope_append_fp4(ctx, dtype, hq, P(x), ld, ctypes.byref(c), ctypes.byref(b), layout, rot, P(table), n_table, P(Q), ldq, P(None))]

    def rows(dtype=0, K=x, ldk=128, V=x + 4096, ldv=128, **kw):
        c, b = structs(**kw)
        return g.STATUS_NAMES[lib.gelo_cache_rows_fp4(ctx, dtype, ctypes.byref(c), ctypes.byref(b), P(K), ldk, P(V), ldv, P(None))]

    def attend(dtype=0, hq=4, Q=x, ldq=256, scale=0.125, O=x, ldo=256, **kw):
        c, b = structs(**kw)
        return g.STATUS_NAMES[lib.gelo_attention_fp4(ctx, dtype, hq, P(Q), ldq, ctypes.byref(c), ctypes.byref(b), scale, 1, P(O), ldo, P(None))]
    for call in (append, rows, attend):
        for bad in ({"k": None}, {"v": None}, {"n_pages": 0}, {"n_kv_heads": 0}, {"page_rows": 0}, {"head_dim": 0}, {"head_stride": piece - 16}, {"page_stride": 16},
                    {"n_seqs": 0}, {"n_rows": 0}, {"max_rows": 0}, {"max_kv_len": 0}, {"kv_len": None}, {"page_table": None}, {"n_rows": 3}, {"max_rows": 2}, {"dtype": 3}):
            assert call(**bad) == "GELO_EINVAL", bad
        for bad in ({"page_rows": 8}, {"page_rows": 48}, {"head_dim": 48}, {"page_rows": 1 << 24}, {"page_stride": 1 << 31}, {"table_ld": 1}, {"max_kv_len": 33}, {"row_start": i, "n_rows": (1 << 22) + 1}):
            assert call(**bad) == "GELO_ESHAPE", bad
        for bad in ({"k": x + 8}, {"head_stride": piece + 8}, {"page_stride": 2 * piece + 4}, {"kv_len": i + 2}, {"page_table": i + 1}):
            assert call(**bad) == "GELO_EALIGN", bad
    for bad in ({"hq": -1}, {"Q": None}, {"hq": 0}, {"ld": 504}, {"layout": 2}, {"rot": 24}, {"rot": 80}, {"table": None}, {"Q": x + 64}):
        assert append(**bad) == "GELO_EINVAL", bad
    assert append(n_table=31) == "GELO_ESHAPE" and append(table=x + 4) == append(ldq=260) == "GELO_EALIGN"
    for bad in ({"K": None, "V": None}, {"ldk": 120}, {"ldv": 120}, {"V": x + 16}):
        assert rows(**bad) == "GELO_EINVAL", bad
    assert rows(K=x + 4) == rows(ldv=132) == "GELO_EALIGN"
    for bad in ({"hq": 0}, {"hq": 3}, {"Q": None}, {"O": None}, {"ldq": 248}, {"scale": float("nan")}, {"scale": float("inf")}, {}):
        assert attend(**bad) == "GELO_EINVAL", bad
    assert attend(head_dim=32, O=x + 8192) == "GELO_ESHAPE" and attend(O=x + 4) == attend(ldo=260) == "GELO_EALIGN"
    torch.cuda.synchronize()
    assert torch.all(buf == 5)
