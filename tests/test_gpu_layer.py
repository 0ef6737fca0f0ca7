"""Norm, rotary positions with the paged cache, and attention, through the C ABI, against the float64 reference.

Bounds, element by element, from the formats' unit roundoffs U32 = 2^-24 and U16 = 2^-8 (bfloat16): see each test.  None is fitted to a
result."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
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


# ---------------------------------------------------------------------------------------------------------- norm --
NORM_SIZES = [(1, 8), (1, 4096), (3, 72), (5, 512), (64, 520), (7, 776), (2, 2048), (65, 2056), (3, 4104), (2, 8192), (3, 8200), (2, 16392), (1, 65536)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d", NORM_SIZES)
def test_norm(ctx, n, d, dtype):
    """A thread adds up to 64 squares, a row 6 + 16 more sums, all positive: at most 90 U32 of the sum, half of that in its root; the
    root, h itself, the division and two products add a few: 64 U32 of |y|.  bfloat16: one rounding more."""
    x, r = rand((n, d), d, dtype, 3.0), rand((n, d), d + 1, dtype)
    gamma = (1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(d + 2))).to(dtype).cuda()
    u = U16 if dtype == BF16 else 0.0
    for residual in (None, r):
        H, H_all = padded(n, d, d + 8, dtype)
        R, R_all = padded(n, d, d + 16, dtype)
        codes = torch.full((n, (d + 15) // 16 * 16 + 16), 9, dtype=torch.uint8, device="cuda")
        scales = torch.full((n,), 5.0, device="cuda")
        g.gelo_rms_norm(ctx, x, gamma, 1e-5, H=H, residual=residual, residual_out=R, codes=codes[:, :d], scales=scales)
        h, y = lo.rms_norm(host(x), host(gamma), 1e-5, None if residual is None else host(residual))
        within(R, h, (U32 + u) * np.abs(h) * 1.01, "residual")
        within(H, y, (64 * U32 + u) * np.abs(y) * 1.01 + 1e-38, "H")
        assert torch.all(H_all[:, d:] == 7) and torch.all(R_all[:, d:] == 7) and torch.all(codes[:, d:] == 9)
        top = np.abs(y).max(1)
        within(scales, top / 448, 70 * U32 * top / 448)
        # the grid of E4M3: half a step is 2^-4 of a normal value at most, 2^-10 below 2^-6
        t = y / host(scales)[:, None]
        c = codes[:, :d].contiguous().view(torch.float8_e4m3fn)
        within(c, t, np.maximum(2.0 ** -4 * np.abs(t), 2.0 ** -10) + 256 * U32 * np.abs(t) + 1e-12, "codes")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_in_place_and_through_strides(ctx, dtype):
    n, d = 37, 264
    x, r, gamma = rand((n, d), 1, dtype), rand((n, d), 2, dtype), rand((d,), 3, dtype)
    want_h, want_r = torch.empty_like(x), torch.empty_like(x)
    g.gelo_rms_norm(ctx, x, gamma, 1e-6, H=want_h, residual=r, residual_out=want_r)
    wide = torch.zeros((n, 3 * d), dtype=dtype, device="cuda")
    X, R = wide[:, d:2 * d], r.clone()
    X.copy_(x)
    g.gelo_rms_norm(ctx, X, gamma, 1e-6, H=X, residual=R, residual_out=R)
    assert torch.equal(X, want_h) and torch.equal(R, want_r)
    assert torch.all(wide[:, :d] == 0) and torch.all(wide[:, 2 * d:] == 0)


def test_norm_of_rows_with_nothing_or_not_a_number(ctx):
    x = rand((5, 512), 4, BF16)
    x[1] = 0
    x[2, 100] = float("nan")
    x[3, 7] = float("inf")
    gamma = torch.ones(512, dtype=BF16, device="cuda")
    H, codes, scales = torch.empty_like(x), torch.empty((5, 512), dtype=torch.uint8, device="cuda"), torch.empty(5, device="cuda")
    g.gelo_rms_norm(ctx, x, gamma, 1e-5, H=H, codes=codes, scales=scales)
    assert torch.all(H[1] == 0) and scales[1] == 1 and torch.all(codes[1] & 0x7F == 0)
    assert torch.isnan(H[2]).all() and torch.isnan(scales[2]) and torch.all(codes[2] == 0x7F)
    assert torch.isnan(H[3, 7]) and torch.all(H[3, :7] == 0) and torch.isnan(scales[3])
    assert torch.isfinite(H[[0, 4]].float()).all() and torch.isfinite(scales[[0, 4]]).all()


def test_codes_feed_the_8_bit_projection(ctx):
    """gelo_project_fp8 is the row quantisation and gelo_project_fp8_codes on its result, bit for bit; with the norm's own codes the product
    stays within the 8-bit grid: relative error 2^-4 of each factor at worst, about a third of it in the Frobenius norm."""
    n, d, p = 130, 256, 264
    X, W = rand((n, d), 5, BF16), rand((d, p), 6, BF16, 0.05)
    Wq = g.gelo_prepare_weight_fp8(ctx, W)
    Y, Z = torch.empty((n, p), dtype=BF16, device="cuda"), torch.empty((n, p), dtype=BF16, device="cuda")
    g.gelo_project_fp8(ctx, X, Wq, p, Y)
    codes, scales = g.gelo_debug_quantize_rows_fp8(ctx, X)
    g.gelo_project_fp8_codes(ctx, codes, scales, Wq, p, Z)
    assert torch.equal(Y, Z)
    gamma = torch.ones(d, dtype=BF16, device="cuda")
    wide = torch.empty((n, d + 32), dtype=torch.uint8, device="cuda")
    g.gelo_rms_norm(ctx, X, gamma, 1e-5, codes=wide[:, :d], scales=scales)
    g.gelo_project_fp8_codes(ctx, wide[:, :d], scales, Wq, p, Z)
    want = lo.rms_norm(host(X), host(gamma), 1e-5)[1] @ host(W)
    assert np.linalg.norm(host(Z) - want) < 2 * 2.0 ** -4 * np.linalg.norm(want)


# ---------------------------------------------------------------------------------------------------------- rope --
@pytest.mark.parametrize("rot,kw", [(16, {}), (128, {}), (64, {"factor": 4.0}), (128, {"base": 5e5, "factor": 8.0, "trained": 8192.0}), (96, {"first_pos": 100000})])
def test_rope_table(ctx, rot, kw):
    """Angles in double: what is left is the rounding to float, half a unit of a value up to 1, and 1e-9 of an angle up to 1e5."""
    table = g.gelo_rope_table(ctx, rot, 301, **kw)
    first = kw.pop("first_pos", 0)
    angles = np.outer(first + np.arange(301), lo.rope_frequencies(rot, **kw))
    within(table[..., 0], np.cos(angles), U32 / 2 + 2e-9)
    within(table[..., 1], np.sin(angles), U32 / 2 + 2e-9)


def make_cache(n_pages, heads, page, d, dtype, order, fill=None, seed=0):
    shape = (n_pages, heads, page, d) if order == "head" else (n_pages, page, heads, d)
    if fill is None:
        K, V = rand(shape, seed, dtype), rand(shape, seed + 1, dtype)
    else:
        K, V = (torch.full(shape, fill, dtype=dtype, device="cuda") for _ in range(2))
    return (K, V) if order == "head" else (K.permute(0, 2, 1, 3), V.permute(0, 2, 1, 3))


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


APPENDS = [  # dtype, new rows, rows in the cache with them, q heads, kv heads, d, page, order, rot, pairs
    (BF16, [1, 1, 1], [1, 16, 17], 4, 4, 64, 16, "head", 64, False),
    (BF16, [5, 0, 33, 1], [5, 9, 40, 64], 6, 2, 128, 32, "row", 64, True),
    (F32, [2, 31], [130, 31], 5, 5, 96, 64, "row", 96, False),
    (F32, [17], [20], 2, 1, 256, 16, "head", 16, True),
    (BF16, [70], [70], 7, 1, 80, 128, "head", 48, False),
    (BF16, [9, 12], [9, 12], 0, 3, 64, 16, "head", 0, False),
]


@pytest.mark.parametrize("dtype,new,kv,hq,hkv,d,page,order,rot,pairs", APPENDS)
def test_append(ctx, dtype, new, kv, hq, hkv, d, page, order, rot, pairs):
    """A turned component is two products and a sum of cosines off by U32: 4 U32 (|a| + |b|), and in bfloat16 one rounding; the rest is
    copied bit for bit and nothing else in the cache moves."""
    batch, table, row_start, n_pages = make_batch(new, kv, page, 1)
    rows = int(row_start[-1])
    K, V = make_cache(n_pages, hkv, page, d, dtype, order, fill=3.0)
    QKV, _ = padded(rows, (hq + 2 * hkv) * d, (hq + 2 * hkv) * d + 8, dtype)
    QKV.copy_(rand(QKV.shape, 2, dtype))
    Q, Q_all = padded(rows, hq * d, hq * d + 24, dtype) if hq else (None, None)
    cs = g.gelo_rope_table(ctx, rot, max(kv)) if rot else None
    g.gelo_rope_append(ctx, QKV, hq, g.KvCache(K, V), batch, Q=Q, table=cs, rot_dim=rot, layout=g.GELO_ROPE_PAIRS if pairs else g.GELO_ROPE_HALF)
    x = host(QKV).reshape(rows, hq + 2 * hkv, d)
    w = lo.rope_frequencies(rot) if rot else np.zeros(0)
    wantK, wantV, wantQ = np.full(K.shape, 3.0), np.full(V.shape, 3.0), np.zeros((rows, hq, d))
    slackK, slackQ = np.zeros(K.shape), np.zeros((rows, hq, d))
    u = U16 if dtype == BF16 else 0.0
    for s in range(len(kv)):
        for j in range(new[s]):
            row, p = row_start[s] + j, kv[s] - new[s] + j
            turned = lo.rotate(x[row, :hq + hkv], w * p, pairs)
            first = np.arange(rot // 2) * 2 if pairs else np.arange(rot // 2)
            second = first + 1 if pairs else first + rot // 2
            slack = np.zeros(turned.shape)
            size = np.abs(x[row, :hq + hkv][:, first]) + np.abs(x[row, :hq + hkv][:, second])
            slack[:, first] = 4 * U32 * size + 1.01 * u * np.abs(turned[:, first])
            slack[:, second] = 4 * U32 * size + 1.01 * u * np.abs(turned[:, second])
            at, r = table[s, p // page], p % page
            wantQ[row], slackQ[row] = turned[:hq], slack[:hq]
            wantK[at, :, r], slackK[at, :, r], wantV[at, :, r] = turned[hq:], slack[hq:], x[row, hq + hkv:]
    within(K, wantK, slackK, "K")
    within(V, wantV, 0.0, "V")
    if hq:
        within(Q.reshape(rows, hq, d), wantQ, slackQ, "Q")
        assert torch.all(Q_all[:, hq * d:] == 7)
        Kp, Vp = make_cache(n_pages, hkv, page, d, dtype, order, fill=3.0)       # in place: the queries turn where they lie
        before = QKV.clone()
        g.gelo_rope_append(ctx, QKV, hq, g.KvCache(Kp, Vp), batch, Q=QKV[:, :hq * d], table=cs, rot_dim=rot,
                           layout=g.GELO_ROPE_PAIRS if pairs else g.GELO_ROPE_HALF)
        assert torch.equal(QKV[:, :hq * d], Q) and torch.equal(QKV[:, hq * d:], before[:, hq * d:])
        assert torch.equal(Kp, K) and torch.equal(Vp, V)


def test_rows_that_have_no_place(ctx):
    """A position below zero, one at the bound, a page number outside the cache, a row of no sequence."""
    page, d = 16, 64
    K, V = make_cache(4, 1, page, d, BF16, "head", fill=3.0)
    table = torch.tensor([[0, 1], [2, 3], [4, -1], [-7, 0]], dtype=torch.int32, device="cuda")
    kv = torch.tensor([1, 33, 5, 7], dtype=torch.int32, device="cuda")
    row_start = torch.tensor([0, 2, 4, 5, 6], dtype=torch.int32, device="cuda")
    batch = g.SeqBatch(kv, table, 32, row_start=row_start, max_rows=2)
    QKV = rand((8, 3 * d), 3, BF16)
    Q = torch.full((8, d), 7.0, dtype=BF16, device="cuda")
    g.gelo_rope_append(ctx, QKV, 1, g.KvCache(K, V), batch, Q=Q)
    assert torch.all(Q[0] == 0)                                        # position -1
    assert torch.equal(Q[1], QKV[1, :d]) and torch.equal(K[0, 0, 0], QKV[1, d:2 * d])
    assert torch.equal(Q[2], QKV[2, :d]) and torch.equal(V[3, 0, 15], QKV[2, 2 * d:])
    assert torch.isnan(Q[3]).all()                                     # position 32 = max_kv_len
    assert torch.equal(Q[4:6], QKV[4:6, :d])                           # pages 4 and -7: not there, not written
    assert torch.all(Q[6:] == 7)
    touched = torch.zeros_like(K, dtype=torch.bool)
    touched[0, 0, 0] = touched[3, 0, 15] = True
    assert torch.all(K[~touched] == 3) and torch.all(V[~touched] == 3)


# ----------------------------------------------------------------------------------------------------- attention --
def attention_bound(ref, absolute, Q, K, scale, kv, d, dtype):
    """A score is a sum of d products, scaled: (d + 6) U32 of |q| |k| scale, which the exponential makes a relative error of its weight; the sums
    over the keys err by a U32 per key and rescaling; all of it twice (weights and their sum) on sum w |v|.  bfloat16: every
    weight rounded, in their sum too, which is U16 of sum w |v - O|, at most that of sum w |v| + |O|; the result rounded once."""
    q = np.linalg.norm(Q.reshape(-1, d), axis=1).max()
    k = np.linalg.norm(np.nan_to_num(K, nan=0.0, posinf=0.0, neginf=0.0).reshape(-1, d), axis=1).max()
    e = U32 * ((d + 6) * abs(scale) * q * k + kv + 64)
    bound = 2 * e * absolute
    if dtype == BF16:
        bound = bound + 1.01 * U16 * (absolute + 2 * np.abs(ref))
    return bound + 1e-30


def run_attention(ctx, dtype, new, kv, hq, hkv, d, page, order, causal, scale=None, max_kv=None, one_row=False, seed=7, stale=float("nan")):
    """Everything that no query may see - rows behind a sequence's end, pages of nobody - holds `stale`."""
    batch, table, row_start, n_pages = make_batch(new, kv, page, seed, max_kv=max_kv, one_row=one_row)
    rows = int(row_start[-1])
    K, V = make_cache(n_pages, hkv, page, d, dtype, order, seed=seed + 1)
    hidden = torch.ones((n_pages, page), dtype=torch.bool)
    for s, n in enumerate(kv):
        for p in range(n):
            hidden[table[s, p // page], p % page] = False
    hidden = hidden.cuda()[:, None, :, None]
    K.masked_fill_(hidden, stale)
    V.masked_fill_(hidden, stale)
    Q, _ = padded(rows, hq * d, hq * d + 40, dtype)
    Q.copy_(rand(Q.shape, seed + 3, dtype))
    O, O_all = padded(rows, hq * d, hq * d + 16, dtype)
    scale = 1 / math.sqrt(d) if scale is None else scale
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, scale, causal=causal)
    assert torch.all(O_all[:, hq * d:] == 7)
    ref, absolute = lo.attention(host(Q), host(K), host(V), hq, row_start, kv, table, scale, causal)
    within(O, ref, attention_bound(ref, absolute, host(Q), host(K), scale, max(kv), d, dtype))
    return O, ref


DECODES = [  # kv, q heads, kv heads, d, page, order
    ([1], 1, 1, 64, 16, "head"),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33], 4, 4, 128, 16, "head"),
    ([127, 128, 129, 255, 256, 257, 0], 6, 2, 64, 64, "row"),
    ([300, 5], 14, 2, 96, 32, "row"),
    ([77, 1030], 16, 1, 256, 16, "head"),
    ([513, 40], 48, 2, 64, 128, "head"),
    ([2100], 8, 8, 128, 64, "row"),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kv,hq,hkv,d,page,order", DECODES)
def test_attention_of_single_tokens(ctx, dtype, kv, hq, hkv, d, page, order):
    run_attention(ctx, dtype, [1] * len(kv), kv, hq, hkv, d, page, order, True, one_row=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("order", ["row", "head"])
def test_single_tokens_of_many_sequences(ctx, dtype, order):
    """So many sequences and heads that a wave has a head of its own where the heads' rows lie side by side; lengths at the edges of tiles."""
    kv = [0, 1, 15, 16, 17, 31, 32, 33, 100, 127, 128, 129] * 11
    run_attention(ctx, dtype, [1] * len(kv), kv, 16, 16, 64, 16, order, True, one_row=True, seed=2)
    run_attention(ctx, dtype, [1] * len(kv), kv, 48, 16, 96, 32, order, True, one_row=True, seed=2)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_where_the_bound_is_far_above_the_lengths(ctx, dtype):
    """A captured launch is sized for the longest context: chunks that no sequence reaches."""
    run_attention(ctx, dtype, [1] * 3, [3, 700, 0], 4, 2, 128, 16, "head", True, one_row=True, max_kv=9000)


PROMPTS = [  # new rows, kv, q heads, kv heads, d, page, order, causal
    ([1, 5], [1, 5], 2, 2, 64, 16, "head", True),
    ([16, 17, 0, 33], [16, 17, 4, 33], 4, 1, 128, 16, "row", True),
    ([64, 65], [64, 200], 2, 2, 128, 64, "head", True),
    ([3, 20], [2, 7], 3, 3, 64, 32, "head", True),              # more new rows than the cache holds: the first ones see nothing
    ([129], [129], 3, 1, 96, 16, "head", True),
    ([130, 40], [700, 41], 4, 2, 64, 32, "row", True),
    ([31, 70], [33, 71], 2, 1, 256, 16, "head", True),
    ([257], [300], 5, 5, 128, 128, "row", True),
    ([2], [1500], 8, 1, 128, 16, "head", True),
    ([5, 33, 12], [1, 100, 0], 4, 4, 64, 16, "head", False),     # cross attention, one sequence without states
    ([70, 200], [257, 64], 2, 2, 128, 64, "row", False),
    ([9], [130], 12, 2, 96, 32, "head", False),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new,kv,hq,hkv,d,page,order,causal", PROMPTS)
def test_attention_of_prompts(ctx, dtype, new, kv, hq, hkv, d, page, order, causal):
    run_attention(ctx, dtype, new, kv, hq, hkv, d, page, order, causal)


LARGE = [  # dtype, new rows, kv, q heads, kv heads, d, page, order, causal
    (BF16, [512, 377, 512, 1, 130, 512, 256, 400], [512, 377, 600, 1, 130, 512, 256, 400], 32, 32, 128, 16, "head", True),      # tiles of columns in pairs
    (BF16, [384, 200, 384, 384, 129, 384, 300, 384], [384, 200, 384, 500, 129, 384, 300, 384], 32, 32, 128, 64, "row", True),   # ... of an odd number
    (BF16, [384, 130, 384, 70], [384, 130, 390, 70], 32, 32, 256, 32, "head", True),
    (BF16, [390, 128] * 4, [390, 300] * 4, 32, 32, 64, 16, "row", True),
    (BF16, [200], [5000], 8, 8, 64, 64, "head", True),                  # many columns and a cut cache
    (BF16, [65, 200], [3000, 4111], 12, 4, 96, 16, "row", False),
    (BF16, [90], [7000], 16, 4, 128, 32, "head", True),
    (BF16, [300, 20], [2500, 90], 8, 4, 256, 16, "head", True),
    (BF16, [1500], [2777], 14, 2, 128, 128, "row", True),
    (BF16, [1, 1], [30011, 9], 16, 2, 128, 64, "head", True),           # few columns and many cuts
    (F32, [1], [20000], 8, 2, 96, 16, "row", True),
    (F32, [700, 33], [1300, 33], 8, 2, 128, 64, "head", True),
    (BF16, [1, 1, 1], [4100, 3000, 1], 48, 2, 64, 32, "head", True),    # more than 16 heads to a key head
]


@pytest.mark.parametrize("dtype,new,kv,hq,hkv,d,page,order,causal", LARGE)
def test_attention_at_the_sizes_where_launches_differ(ctx, dtype, new, kv, hq, hkv, d, page, order, causal):
    """The reference in float64 on the GPU, for every sequence and two of the heads; the same bound as above."""
    batch, table, row_start, n_pages = make_batch(new, kv, page, 3, one_row=max(new) == 1)
    rows = int(row_start[-1])
    K, V = make_cache(n_pages, hkv, page, d, dtype, order, seed=5)
    Q, O = rand((rows, hq * d), 8, dtype), torch.full((rows, hq * d), 7.0, dtype=dtype, device="cuda")
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d), causal=causal)
    assert torch.isfinite(O.float()).all()
    for s in range(len(kv)):
        used = torch.from_numpy(table[s, :(kv[s] + page - 1) // page]).long().cuda()
        at = slice(int(row_start[s]), int(row_start[s + 1]))
        for h in {0, (7 * s + 5) % hq}:
            kh = h * hkv // hq
            k, v = (x[used, kh].reshape(-1, d)[:kv[s]].double() for x in (K, V))
            q = Q[at, h * d:(h + 1) * d].double()
            score = q @ k.T / math.sqrt(d)
            if causal:
                score.masked_fill_(torch.arange(kv[s], device="cuda")[None] > torch.arange(new[s], device="cuda")[:, None] + (kv[s] - new[s]), -math.inf)
            w = torch.softmax(score, -1)
            ref, absolute = host(w @ v), host(w @ v.abs())
            within(O[at, h * d:(h + 1) * d], ref, attention_bound(ref, absolute, host(q), host(k), 1 / math.sqrt(d), kv[s], d, dtype), (s, h))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_attention_scales(ctx, dtype, scale):
    """Equal weights, reversed ones, and scores so far apart that a single key is left."""
    run_attention(ctx, dtype, [1, 20], [90, 150], 4, 2, 64, 16, "head", True, scale=scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(ctx, dtype, d, value):
    new, page, at = 150, 16, 75
    K, V = make_cache(12, 1, page, d, dtype, "head", seed=3)
    V[at // page, 0, at % page, 5] = value
    K[at // page, 0, at % page] = 0
    table = torch.arange(12, dtype=torch.int32, device="cuda")[None]
    batch = g.SeqBatch(torch.tensor([new], dtype=torch.int32).cuda(), table, new, row_start=torch.tensor([0, new], dtype=torch.int32).cuda(), max_rows=new)
    Q = rand((new, d), 9, dtype)
    O = torch.empty_like(Q)
    g.gelo_attention(ctx, Q, O, 1, g.KvCache(K, V), batch, 1 / math.sqrt(d))
    clean = V.clone()
    clean[at // page, 0, at % page, 5] = 0
    want = torch.empty_like(Q)
    g.gelo_attention(ctx, Q, want, 1, g.KvCache(K, clean), batch, 1 / math.sqrt(d))
    other = torch.arange(d, device="cuda") != 5
    assert torch.equal(O[:, other], want[:, other]) and torch.equal(O[:at], want[:at])
    assert torch.isfinite(want.float()).all()
    assert torch.isnan(O[at:, 5]).all() if math.isnan(value) else torch.all(O[at:, 5] == value)
    # a key that is NaN: the rows before it do not see it
    K[at // page, 0, at % page, 0] = float("nan")
    g.gelo_attention(ctx, Q, O, 1, g.KvCache(K, clean), batch, 1 / math.sqrt(d))
    assert torch.equal(O[:at], want[:at]) and torch.isnan(O[at:]).all()


def way(ctx, Q, new, kv, hq, hkv, d, causal):
    """Which way such a bfloat16 call goes (1: the kernel for many columns to a key head, the cache whole)."""
    return ctypes.CDLL(g.LIB_PATH)["_ZN4gelo13attention_wayEiiiiiiiii"](1, int(causal), hq, hkv, d, len(kv), Q.shape[0], max(new), max(kv))


EDGES = [(1, 1), (5, 1), (16, 16), (17, 17), (31, 40), (32, 32), (33, 63), (63, 64), (64, 65), (65, 64), (127, 128), (128, 127), (129, 200), (2, 0), (0, 9),
         (140, 15), (64, 191), (96, 192), (130, 193), (20, 257), (257, 300), (48, 48), (200, 112), (70, 129)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,hq,hkv,page,order", [(64, 32, 16, 16, "head"), (96, 16, 16, 32, "row"), (128, 32, 16, 16, "row"), (256, 16, 16, 64, "head")])
def test_many_columns_at_the_edges_of_tiles(ctx, d, hq, hkv, page, order, causal):
    """New rows and lengths at, before and behind the ends of tiles, steps and groups, none, and more rows than keys; rows of the cache that
    belong to nobody hold NaN.  All rows of three heads."""
    new, kv = [x[0] for x in EDGES], [x[1] for x in EDGES]
    batch, table, row_start, n_pages = make_batch(new, kv, page, 3)
    K, V = make_cache(n_pages, hkv, page, d, BF16, order, seed=5)
    hidden = torch.ones((n_pages, page), dtype=torch.bool)
    for s, n in enumerate(kv):
        for p in range(n):
            hidden[table[s, p // page], p % page] = False
    K.masked_fill_(hidden.cuda()[:, None, :, None], float("nan"))
    V.masked_fill_(hidden.cuda()[:, None, :, None], float("nan"))
    Q = rand((int(row_start[-1]), hq * d), 8, BF16)
    O = torch.full_like(Q, 7.0)
    assert way(ctx, Q, new, kv, hq, hkv, d, causal) == 1
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d), causal=causal)
    for h in (0, hq // 2 + 1, hq - 1):
        kh = h * hkv // hq
        ref, absolute = lo.attention(host(Q[:, h * d:(h + 1) * d]), host(K[:, kh:kh + 1]), host(V[:, kh:kh + 1]), 1, row_start, kv, table, 1 / math.sqrt(d), causal)
        within(O[:, h * d:(h + 1) * d], ref, attention_bound(ref, absolute, host(Q), host(K), 1 / math.sqrt(d), max(kv), d, BF16), h)


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_many_columns_at_other_scales(ctx, scale):
    new, kv, hq, d, page = [150] * 16, [150 + 9 * i for i in range(16)], 16, 128, 16
    batch, table, row_start, n_pages = make_batch(new, kv, page, 3)
    K, V = make_cache(n_pages, hq, page, d, BF16, "head", seed=5)
    Q = rand((int(row_start[-1]), hq * d), 8, BF16)
    O = torch.full_like(Q, 7.0)
    assert way(ctx, Q, new, kv, hq, hq, d, True) == 1
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, scale)
    for h in (0, hq - 1):
        ref, absolute = lo.attention(host(Q[:, h * d:(h + 1) * d]), host(K[:, h:h + 1]), host(V[:, h:h + 1]), 1, row_start, kv, table, scale, True)
        within(O[:, h * d:(h + 1) * d], ref, attention_bound(ref, absolute, host(Q), host(K), scale, max(kv), d, BF16), h)


@pytest.mark.parametrize("rows,want", [(150, 1), (512, 2)])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_many_columns_and_values_that_are_not_finite(ctx, d, value, rows, want):
    """One component of one value in every sequence and head: only rows from its own on, and only that component; everything else keeps its
    bits.  A key that is NaN: the rows before it do not see it.  A page number outside the cache: its sequence alone."""
    n_seqs, hq = (8 if d == 256 else 16), 16               # (at this width a workgroup has a CU to itself: half as many fit)
    rows = 384 if want == 2 and d == 256 else rows
    page, at = 16, 75
    each = (rows + page - 1) // page
    K, V = make_cache(n_seqs * each, hq, page, d, BF16, "head", seed=3)
    table = torch.arange(n_seqs * each, dtype=torch.int32, device="cuda").view(n_seqs, each)
    pages = table[:, at // page].long()
    K[pages, :, at % page] = 0
    odd = V.clone()
    odd[pages, :, at % page, 5] = value
    V[pages, :, at % page, 5] = 0
    row_start = (torch.arange(n_seqs + 1, device="cuda") * rows).int()
    batch = g.SeqBatch(torch.full((n_seqs,), rows, dtype=torch.int32).cuda(), table, rows, row_start=row_start, max_rows=rows)
    Q = rand((n_seqs * rows, hq * d), 9, BF16)
    assert way(ctx, Q, [rows] * n_seqs, [rows] * n_seqs, hq, hq, d, True) == want
    O, clean = torch.empty_like(Q), torch.empty_like(Q)
    g.gelo_attention(ctx, Q, clean, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d))
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, odd), batch, 1 / math.sqrt(d))
    o, w = (x.view(n_seqs, rows, hq, d) for x in (O, clean))
    other = torch.arange(d, device="cuda") != 5
    assert torch.isfinite(w.float()).all()
    assert torch.equal(o[..., other], w[..., other]) and torch.equal(o[:, :at], w[:, :at])
    assert torch.isnan(o[:, at:, :, 5]).all() if math.isnan(value) else torch.all(o[:, at:, :, 5] == value)
    K[pages, :, at % page, 0] = float("nan")
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d))
    assert torch.equal(o[:, :at], w[:, :at]) and torch.isnan(o[:, at:]).all()
    K[pages, :, at % page, 0] = 0
    table[3, 2] = n_seqs * each
    table[7, 0] = -3
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d))
    assert torch.isnan(o[7]).all() and torch.isnan(o[3, -1]).all()
    rest = [s for s in range(n_seqs) if s not in (3, 7)]
    assert torch.equal(o[rest], w[rest])


@pytest.mark.parametrize("d", [64, 128])
def test_a_cut_cache_and_values_that_are_not_finite(ctx, d):
    """Many columns, the keys in chunks whose parts are joined: the value lies in one chunk."""
    rows, kv, hq, page, at = 200, 5000, 8, 64, 4900
    K, V = make_cache(79, hq, page, d, BF16, "row", seed=3)
    table = torch.arange(79, dtype=torch.int32, device="cuda")[None]
    batch = g.SeqBatch(torch.tensor([kv], dtype=torch.int32).cuda(), table, kv, row_start=torch.tensor([0, rows], dtype=torch.int32).cuda(), max_rows=rows)
    Q = rand((rows, hq * d), 9, BF16)
    assert way(ctx, Q, [rows], [kv], hq, hq, d, True) == 5
    K[at // page, :, at % page] = 0
    V[at // page, :, at % page, 5] = 0
    O, clean = torch.empty_like(Q), torch.empty_like(Q)
    g.gelo_attention(ctx, Q, clean, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d))
    V[at // page, :, at % page, 5] = float("inf")
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d))
    o, w = (x.view(rows, hq, d) for x in (O, clean))
    first, other = at - (kv - rows), torch.arange(d, device="cuda") != 5
    assert torch.equal(o[..., other], w[..., other]) and torch.equal(o[:first], w[:first]) and torch.all(o[first:, :, 5] == float("inf"))


# the ways are the numbers of `way`; float goes through the one kernel it has
NO_SOFTMAX = [(F32, [1, 1], [300, 0], 4, 64, None), (F32, [40, 7], [40, 1500], 2, 128, None), (BF16, [1, 1], [200, 0], 4, 96, 0),
              (BF16, [1, 1], [9000, 0], 4, 128, 4), (BF16, [150] * 14 + [3], [150] * 14 + [0], 16, 128, 1),
              (BF16, [150] * 16 + [3], [150] * 16 + [0], 16, 96, 2), (BF16, [200, 4], [4096, 0], 4, 64, 5)]


@pytest.mark.parametrize("dtype,new,kv,hq,d,want", NO_SOFTMAX)
def test_a_row_that_sees_only_scores_of_minus_infinity_has_no_softmax(ctx, dtype, new, kv, hq, d, want):
    """exp(-inf - max) / sum is 0 / 0 there: NaN, unlike the zeros of a row that sees no key.  The other rows and heads do not notice."""
    page = 16
    batch, table, row_start, n_pages = make_batch(new, kv, page, 3)
    K, V = make_cache(n_pages, hq, page, d, dtype, "head", seed=5)
    K[..., 0] = K[..., 0].abs() + 0.125
    rows = int(row_start[-1])
    Q = rand((rows, hq * d), 8, dtype)
    row, head = min(rows - 1, 33) if new[0] > 1 else 0, hq - 1
    Q[row, head * d] = -math.inf
    O = torch.full_like(Q, 7.0)
    if want is not None:
        assert way(ctx, Q, new, kv, hq, hq, d, True) == want
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d))
    there = torch.isnan(O).view(rows, hq, d)
    assert there[row, head].all() and there.sum() == d
    for s, n in enumerate(kv):
        if n == 0:
            assert torch.all(O[int(row_start[s]):int(row_start[s + 1])] == 0)


@pytest.mark.parametrize("d", [64, 96, 128, 256])
@pytest.mark.parametrize("new,hq,hkv,want", [([1] * 5, 4, 2, 0), ([150] * 16, 16, 16, 1)])
def test_a_row_that_sees_one_key_is_its_value(ctx, new, hq, hkv, want, d):
    """Weight times value over weight, for every weight: the value's own bits, since the same rounded weight stands above and below."""
    new = new[:8] if d == 256 else new                     # (at this width half as many workgroups fit, and more go in pairs)
    batch, table, row_start, n_pages = make_batch(new, [1] * len(new), 16, 3)
    K, V = make_cache(n_pages, hkv, 16, d, BF16, "head", seed=5)
    Q = rand((int(row_start[-1]), hq * d), 8, BF16)
    O = torch.full_like(Q, 7.0)
    assert way(ctx, Q, new, [1] * len(new), hq, hkv, d, False) == want
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d), causal=False)
    heads = torch.arange(hq, device="cuda") * hkv // hq
    for s in range(len(new)):
        assert torch.equal(O[int(row_start[s]):int(row_start[s + 1])].view(-1, hq, d), V[int(table[s, 0]), heads, 0].expand(new[s], hq, d))


def float_way(new, kv, hq, hkv, d, causal):
    """1: float by tiles of 64 columns, 5: with a cut cache."""
    return ctypes.CDLL(g.LIB_PATH)["_ZN4gelo19attention_float_wayEiiiiiiii"](int(causal), hq, hkv, d, len(kv), sum(new), max(new), max(kv))


FLOAT_TILES = [  # new, kv, q heads, kv heads, d, page, order, causal, scale, way
    ([x[0] for x in EDGES], [x[1] for x in EDGES], 16, 16, 96, 16, "row", True, None, 1),
    ([x[0] for x in EDGES], [x[1] for x in EDGES], 32, 16, 128, 32, "head", False, None, 1),
    ([200, 1, 64, 65], [1000, 1, 513, 0], 16, 16, 128, 64, "head", False, None, 5),
    ([65, 17], [700, 300], 64, 8, 96, 16, "row", True, None, 5),
    ([60] * 34, [60 + i for i in range(34)], 16, 16, 128, 16, "head", True, -0.2, 1),
    ([60] * 34, [60 + i for i in range(34)], 16, 16, 96, 16, "head", True, 0.0, 1),
]


@pytest.mark.parametrize("new,kv,hq,hkv,d,page,order,causal,scale,want", FLOAT_TILES)
def test_float_by_tiles_of_64_columns(ctx, new, kv, hq, hkv, d, page, order, causal, scale, want):
    """Edges of tiles and steps, cut caches, rows of the cache that belong to nobody hold NaN; all rows of three heads."""
    batch, table, row_start, n_pages = make_batch(new, kv, page, 3)
    K, V = make_cache(n_pages, hkv, page, d, F32, order, seed=5)
    hidden = torch.ones((n_pages, page), dtype=torch.bool)
    for s, n in enumerate(kv):
        for p in range(n):
            hidden[table[s, p // page], p % page] = False
    K.masked_fill_(hidden.cuda()[:, None, :, None], float("nan"))
    V.masked_fill_(hidden.cuda()[:, None, :, None], float("nan"))
    Q = rand((int(row_start[-1]), hq * d), 8, F32)
    O = torch.full_like(Q, 7.0)
    scale = 1 / math.sqrt(d) if scale is None else scale
    assert float_way(new, kv, hq, hkv, d, causal) == want
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, scale, causal=causal)
    for h in (0, hq // 2 + 1, hq - 1):
        kh = h * hkv // hq
        ref, absolute = lo.attention(host(Q[:, h * d:(h + 1) * d]), host(K[:, kh:kh + 1]), host(V[:, kh:kh + 1]), 1, row_start, kv, table, scale, causal)
        within(O[:, h * d:(h + 1) * d], ref, attention_bound(ref, absolute, host(Q), host(K), scale, max(kv), d, F32), h)


@pytest.mark.parametrize("d", [96, 128])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_float_by_tiles_of_64_columns_and_values_that_are_not_finite(ctx, d, value):
    """One component of one value in every sequence and head, a key that is NaN, a page number outside the cache: as for bfloat16."""
    n_seqs, hq, rows, page, at = 16, 16, 150, 16, 75
    each = (rows + page - 1) // page
    K, V = make_cache(n_seqs * each, hq, page, d, F32, "head", seed=3)
    table = torch.arange(n_seqs * each, dtype=torch.int32, device="cuda").view(n_seqs, each)
    pages = table[:, at // page].long()
    K[pages, :, at % page] = 0
    odd = V.clone()
    odd[pages, :, at % page, 5] = value
    V[pages, :, at % page, 5] = 0
    row_start = (torch.arange(n_seqs + 1, device="cuda") * rows).int()
    kv_len = torch.full((n_seqs,), rows, dtype=torch.int32).cuda()
    batch = g.SeqBatch(kv_len, table, rows, row_start=row_start, max_rows=rows)
    assert float_way([rows] * n_seqs, [rows] * n_seqs, hq, hq, d, True) == 1
    Q = rand((n_seqs * rows, hq * d), 9, F32)
    want, O = torch.empty_like(Q), torch.empty_like(Q)
    g.gelo_attention(ctx, Q, want, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d))
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, odd), batch, 1 / math.sqrt(d))
    o, w = (x.view(n_seqs, rows, hq, d) for x in (O, want))
    assert torch.isfinite(w).all()
    other = torch.arange(d, device="cuda") != 5
    assert torch.equal(o[..., other], w[..., other]) and torch.equal(o[:, :at], w[:, :at])
    seen = o[:, at:, :, 5]
    assert torch.isnan(seen).all() if math.isnan(value) else torch.all(seen == value)
    K[pages, :, at % page, 0] = float("nan")
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, 1 / math.sqrt(d))
    assert torch.equal(o[:, :at], w[:, :at]) and torch.isnan(o[:, at:]).all()
    K[pages, :, at % page, 0] = 0
    bad = table.clone()
    bad[3, 1] = n_seqs * each
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), g.SeqBatch(kv_len, bad, rows, row_start=row_start, max_rows=rows), 1 / math.sqrt(d))
    good = torch.arange(n_seqs, device="cuda") != 3
    assert torch.equal(o[good], w[good]) and torch.isnan(o[3, 64:]).all()


def test_page_numbers_outside_the_cache_are_not_followed(ctx):
    K, V = make_cache(4, 2, 16, 64, BF16, "head", seed=3)
    table = torch.tensor([[0, 1 << 29], [2, 3], [-5, 1]], dtype=torch.int32, device="cuda")
    batch = g.SeqBatch(torch.tensor([20, 20, 20], dtype=torch.int32).cuda(), table, 32)
    Q = rand((3, 128), 9, BF16)
    O = torch.zeros_like(Q)
    g.gelo_attention(ctx, Q, O, 2, g.KvCache(K, V), batch, 0.125)
    assert torch.isnan(O[0]).all() and torch.isnan(O[2]).all() and torch.isfinite(O[1].float()).all()


@pytest.mark.parametrize("new", [1, 70])
def test_a_cache_beyond_32_bit_offsets(ctx, new):
    """Pages whose elements lie behind 2^31: 40000 pages of 16 rows of 16 heads of 256 values are 2.6e9 elements (5.2 GB each)."""
    heads, d, page, n_pages = 16, 256, 16, 40000
    K, V = (torch.zeros((n_pages, heads, page, d), dtype=BF16, device="cuda") for _ in range(2))
    kv = 90
    pages = torch.tensor([[n_pages - 1 - 3 * i for i in range(6)]], dtype=torch.int32, device="cuda")
    batch = g.SeqBatch(torch.tensor([kv], dtype=torch.int32).cuda(), pages, kv, row_start=torch.tensor([0, new], dtype=torch.int32).cuda(), max_rows=new)
    fill = g.SeqBatch(torch.tensor([kv], dtype=torch.int32).cuda(), pages, kv, row_start=torch.tensor([0, kv], dtype=torch.int32).cuda(), max_rows=kv)
    QKV = rand((kv, 3 * heads * d), 5, BF16)
    cache = g.KvCache(K, V)
    whole = torch.empty((kv, heads * d), dtype=BF16, device="cuda")
    g.gelo_rope_append(ctx, QKV, heads, cache, fill, Q=whole)
    small = KVs = [torch.zeros((6, heads, page, d), dtype=BF16, device="cuda") for _ in range(2)]
    near = torch.arange(6, dtype=torch.int32, device="cuda")[None]
    g.gelo_rope_append(ctx, QKV, heads, g.KvCache(*KVs), g.SeqBatch(fill.kv_len, near, kv, row_start=fill.row_start, max_rows=kv), Q=whole)
    assert torch.equal(K[pages[0].long()], small[0]) and torch.equal(V[pages[0].long()], small[1])
    Q = whole[kv - new:].contiguous()
    O, want = torch.empty_like(Q), torch.empty_like(Q)
    g.gelo_attention(ctx, Q, O, heads, cache, batch, 1 / 16)
    g.gelo_attention(ctx, Q, want, heads, g.KvCache(*KVs), g.SeqBatch(batch.kv_len, near, kv, row_start=batch.row_start, max_rows=new), 1 / 16)
    assert torch.equal(O, want) and O.float().abs().sum() > 0


def test_rows_of_no_sequence_are_left_alone(ctx):
    K, V = make_cache(8, 1, 16, 64, BF16, "head", seed=3)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    row_start = torch.tensor([2, 5, 7], dtype=torch.int32).cuda()
    for max_kv in (64, 40):
        batch = g.SeqBatch(torch.tensor([40, 9], dtype=torch.int32).cuda(), table, max_kv, row_start=row_start, max_rows=3)
        Q = rand((10, 64), 9, BF16)
        O = torch.full_like(Q, 7.0)
        g.gelo_attention(ctx, Q, O, 1, g.KvCache(K, V), batch, 0.125)
        assert torch.all(O[:2] == 7) and torch.all(O[7:] == 7) and torch.all(O[2:7] != 7)


def layer(ctx, s):
    g.gelo_rms_norm(ctx, s["X"], s["gamma"], 1e-5, H=s["H"], residual=s["R"], residual_out=s["R_out"])
    g.gelo_rope_append(ctx, s["QKV"], 4, s["cache"], s["batch"], Q=s["Q"], table=s["table"], rot_dim=64)
    g.gelo_attention(ctx, s["Q"], s["O"], 4, s["cache"], s["batch"], 0.125)


def layer_state(ctx, kv, seed):
    batch, _, _, n_pages = make_batch([1] * len(kv), kv, 16, seed, max_kv=3000, one_row=True)
    K, V = make_cache(n_pages, 2, 16, 64, BF16, "head", seed=seed)
    n = len(kv)
    return {"X": rand((n, 256), seed, BF16), "R": rand((n, 256), seed + 1, BF16), "gamma": rand((256,), seed + 2, BF16), "QKV": rand((n, 512), seed + 3, BF16),
            "H": torch.empty((n, 256), dtype=BF16, device="cuda"), "R_out": torch.empty((n, 256), dtype=BF16, device="cuda"),
            "Q": torch.empty((n, 256), dtype=BF16, device="cuda"), "O": torch.empty((n, 256), dtype=BF16, device="cuda"),
            "cache": g.KvCache(K, V), "batch": batch, "table": g.gelo_rope_table(ctx, 64, 3000)}


def test_other_streams_and_captured_graphs(ctx):
    """The three calls on a stream of their own, and captured once and replayed for other inputs in the same buffers, against plain calls."""
    g.gelo_reserve_attention(ctx, 64)
    a = layer_state(ctx, [2500, 40, 7, 0], 20)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        layer(ctx, a)
    side.synchronize()
    O_side, H_side = a["O"].clone(), a["H"].clone()
    a["O"].fill_(3), a["H"].fill_(3)
    layer(ctx, a)
    torch.cuda.synchronize()
    assert torch.equal(a["O"], O_side) and torch.equal(a["H"], H_side)
    assert torch.all(a["O"][3] == 0)                                   # kv_len 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(ctx, a)
    for turn, lens in enumerate(([2500, 40, 7, 0], [2501, 41, 8, 1], [3, 2600, 0, 100], [1, 1, 1, 1])):
        a["QKV"].copy_(rand((4, 512), 50 + turn, BF16))
        a["X"].copy_(rand((4, 256), 60 + turn, BF16))
        pages = torch.arange(4 * 188, dtype=torch.int32).view(4, 188) % a["cache"].K.shape[0]
        a["batch"].page_table.copy_(pages)
        a["batch"].kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        before = a["cache"].K.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = a["O"].clone(), a["H"].clone(), a["cache"].K.clone()
        a["cache"].K.copy_(before)
        layer(ctx, a)
        torch.cuda.synchronize()
        assert torch.equal(a["O"], got[0]) and torch.equal(a["H"], got[1]) and torch.equal(a["cache"].K, got[2])


def test_the_same_call_twice_gives_the_same_bits(ctx):
    O, _ = run_attention(ctx, BF16, [1, 1], [2000, 1111], 8, 2, 128, 16, "head", True, one_row=True)
    again, _ = run_attention(ctx, BF16, [1, 1], [2000, 1111], 8, 2, 128, 16, "head", True, one_row=True)
    assert torch.equal(O, again)


# ------------------------------------------------------------------------------------------------------ refusals --
def status_of(fn, *a, **kw):
    with pytest.raises(g.GeloError) as e:
        fn(*a, **kw)
    return g.STATUS_NAMES[e.value.status]


def test_refusals_of_the_norm(ctx):
    lib, P = g.load_library(), ctypes.c_void_p
    buf = torch.full((4096,), 5.0, device="cuda")
    x = buf.data_ptr()
    def call(dtype=0, n=4, d=64, X=x, ldx=64, R=None, ldr=0, gamma=x, eps=1e-5, Ro=None, ldro=0, H=x, ldh=64, codes=None, ldq=0, scales=None):
        return g.STATUS_NAMES[lib.gelo_rms_norm(ctx, dtype, n, d, P(X), ldx, P(R), ldr, P(gamma), eps, P(Ro), ldro, P(H), ldh, P(codes), ldq, P(scales), P(None))]
    assert g.STATUS_NAMES[lib.gelo_rms_norm(None, 0, 4, 64, P(x), 64, P(None), 0, P(x), 1e-5, P(None), 0, P(x), 64, P(None), 0, P(None), P(None))] == "GELO_EINVAL"
    assert call(dtype=2) == call(n=0) == call(d=0) == call(X=None) == call(gamma=None) == call(H=None) == "GELO_EINVAL"
    assert call(eps=-1.0) == call(eps=float("nan")) == call(eps=float("inf")) == call(ldx=56) == call(codes=x, ldq=64) == "GELO_EINVAL"
    assert call(d=60) == call(X=x + 4) == call(ldx=68) == call(R=x, ldr=68) == call(Ro=x + 8, ldro=64) == call(codes=x, ldq=68, scales=x) == "GELO_EALIGN"
    assert call(d=65544, ldx=65544, ldh=65544) == call(n=(1 << 22) + 1) == "GELO_ESHAPE"
    torch.cuda.synchronize()
    assert torch.all(buf == 5)
    assert b"exceeds" in lib.gelo_last_error(ctx)


def test_refusals_of_the_table_and_the_8_bit_product(ctx):
    lib, P = g.load_library(), ctypes.c_void_p
    buf = torch.full((4096,), 5.0, device="cuda")
    x = buf.data_ptr()
    def table(rot=16, first=0, n=4, base=1e4, factor=1.0, trained=0.0, low=1.0, high=4.0, out=x):
        return g.STATUS_NAMES[lib.gelo_rope_table(ctx, rot, first, n, base, factor, trained, low, high, P(out), P(None))]
    for bad in ({"rot": 0}, {"rot": 24}, {"first": -1}, {"n": 0}, {"first": 2 ** 31 - 2}, {"base": 0.0}, {"base": float("nan")}, {"factor": -1.0},
                {"trained": -1.0}, {"trained": 8.0, "low": 4.0}, {"out": None}):
        assert table(**bad) == "GELO_EINVAL", bad
    assert table(out=x + 4) == "GELO_EALIGN" and table(n=2 ** 30) == "GELO_ESHAPE"
    def codes(n=4, d=128, p=8, c=x, ldq=128, s=x, w=x, y=x, ldy=8):
        return g.STATUS_NAMES[lib.gelo_project_fp8_codes(ctx, n, d, p, P(c), ldq, P(s), P(w), P(y), ldy, P(None))]
    assert codes(n=0) == codes(c=None) == codes(s=None) == codes(w=None) == codes(y=None) == codes(ldq=112) == "GELO_EINVAL"
    assert codes(d=64, ldq=64) == "GELO_ESHAPE" and codes(ldq=136) == codes(c=x + 8) == codes(s=x + 2) == codes(p=12, ldy=16) == "GELO_EALIGN"
    torch.cuda.synchronize()
    assert torch.all(buf == 5)


def test_refusals_of_append_and_attention(ctx):
    lib, P = g.load_library(), ctypes.c_void_p
    buf = torch.full((1 << 16,), 5.0, device="cuda")
    ints = torch.zeros(64, dtype=torch.int32, device="cuda")
    x, i = buf.data_ptr(), ints.data_ptr()
    def structs(**kw):
        c = dict(k=x, v=x, n_pages=2, n_kv_heads=2, page_rows=16, head_dim=64, page_stride=2048, head_stride=1024, row_stride=64)
        b = dict(n_seqs=2, n_rows=2, max_rows=1, max_kv_len=32, row_start=None, kv_len=i, page_table=i, table_ld=2)
        for k, v in kw.items():
            (c if k in c else b)[k] = v
        return g._KvCacheStruct(*c.values()), g._SeqBatchStruct(*b.values())
    def append(dtype=0, hq=4, ld=512, layout=0, rot=64, table=x, n_table=32, Q=x, ldq=256, **kw):
        c, b = structs(**kw)
        return g.STATUS_NAMES[lib.gelo_rope_append(ctx, dtype, hq, P(x), ld, ctypes.byref(c), ctypes.byref(b), layout, rot, P(table), n_table, P(Q), ldq, P(None))]
    def attend(dtype=0, hq=4, Q=x, ldq=256, scale=0.125, O=x, ldo=256, **kw):
        c, b = structs(**kw)
        return g.STATUS_NAMES[lib.gelo_attention(ctx, dtype, hq, P(Q), ldq, ctypes.byref(c), ctypes.byref(b), scale, 1, P(O), ldo, P(None))]
    for call in (append, attend):
        for bad in ({"k": None}, {"v": None}, {"n_pages": 0}, {"n_kv_heads": 0}, {"page_rows": 0}, {"row_stride": 56}, {"head_stride": 0}, {"page_stride": 8},
                    {"n_seqs": 0}, {"n_rows": 0}, {"max_rows": 0}, {"max_kv_len": 0}, {"kv_len": None}, {"page_table": None}, {"n_rows": 3}, {"max_rows": 2}, {"dtype": 3}):
            assert call(**bad) == "GELO_EINVAL", bad
        for bad in ({"page_rows": 8}, {"page_rows": 48}, {"table_ld": 1}, {"max_kv_len": 33}, {"row_stride": (1 << 24) + 8}, {"row_start": i, "n_rows": (1 << 22) + 1}):
            assert call(**bad) == "GELO_ESHAPE", bad
        for bad in ({"k": x + 8}, {"row_stride": 68}, {"head_stride": 1028}, {"kv_len": i + 2}, {"page_table": i + 1}):
            assert call(**bad) == "GELO_EALIGN", bad
    for bad in ({"hq": -1}, {"Q": None}, {"hq": 0}, {"ld": 504}, {"layout": 2}, {"rot": 24}, {"rot": 80}, {"table": None}):
        assert append(**bad) == "GELO_EINVAL", bad
    assert append(n_table=31) == "GELO_ESHAPE" and append(table=x + 4) == append(ldq=260) == "GELO_EALIGN"
    for bad in ({"hq": 0}, {"hq": 3}, {"Q": None}, {"O": None}, {"ldq": 248}, {"scale": float("nan")}, {"scale": float("inf")}):
        assert attend(**bad) == "GELO_EINVAL", bad
    assert attend(head_dim=80, row_stride=80) == "GELO_ESHAPE" and attend(O=x + 4) == attend(ldo=260) == "GELO_EALIGN"
    assert status_of(g.gelo_reserve_attention, ctx, 80) == "GELO_ESHAPE"
    torch.cuda.synchronize()
    assert torch.all(buf == 5)
    # the binding's own checks
    K, V = make_cache(2, 2, 16, 64, BF16, "head")
    with pytest.raises(ValueError):
        g.KvCache(K, V.permute(0, 2, 1, 3))
    with pytest.raises(ValueError):
        g.KvCache(K, V.transpose(2, 3).contiguous().transpose(2, 3))
    with pytest.raises(ValueError):
        g.SeqBatch(torch.zeros(2, dtype=torch.int64, device="cuda"), ints.view(2, 32), 32)
    batch = g.SeqBatch(ints[:2], ints[:4].view(2, 2), 32)
    cache = g.KvCache(K, V)
    Q = torch.zeros((2, 128), dtype=BF16, device="cuda")
    assert status_of(g.gelo_attention, ctx, Q.float(), Q.float(), 2, cache, batch, 1.0) == "GELO_EDTYPE"
    assert status_of(g.gelo_attention, ctx, Q, torch.empty_like(Q), 3, cache, batch, 1.0) == "GELO_ESHAPE"
    three = torch.zeros((3, 128), dtype=BF16, device="cuda")
    assert status_of(g.gelo_attention, ctx, three, torch.empty_like(three), 2, cache, batch, 1.0) == "GELO_ESHAPE"


@pytest.mark.parametrize("dtype,bound", [(BF16, 6e-2), (F32, 3e-4)])
def test_the_layer_example(dtype, bound):
    """Prompts and single tokens through norm, obfuscated projections, cache and attention.  Each of the two projections may be off by its
    contract (2e-2 bf16, 1e-4 float), the first one's error passes attention as it is; norm, rotation and attention round once more each."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_layer.py")
    spec = importlib.util.spec_from_file_location("serve_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    error, _, _ = example.serve(seqs=3, prompt=150, steps=4, dtype=dtype, d=512, q_heads=8, kv_heads=2)
    assert error < bound
