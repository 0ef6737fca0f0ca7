"""The operators between two projections at the limits of what their arguments may hold, through the C ABI."""
import ctypes
import math

import numpy as np
import pytest
import torch

import test_gpu_layer as base
from oracle import layer_oracle as lo
from paper_2603_05035_amd import binding as g
from test_gpu_layer import BF16, F32, U16, U32, attention_bound, float_way, host, make_batch, make_cache, rand, way, within

pytestmark = pytest.mark.gpu

INT_MIN, INT_MAX = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module")
def ctx():
    c = g.gelo_create(0, 1)
    yield c
    g.gelo_destroy(c)


def int32(*values):
    return torch.tensor(values, dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype,hq,hkv,d,many", [(BF16, 2, 2, 64, 0), (BF16, 128, 1, 128, 1), (F32, 2, 2, 96, 0), (F32, 64, 1, 128, 1)])
def test_lengths_and_row_starts_at_the_ends_of_32_bits(ctx, dtype, hq, hkv, d, many):
    """A length below zero is one of zero.  Row starts that do not ascend bring no rows."""
    page, n_seqs, rows = 16, 16, 8
    K, V = make_cache(2 * n_seqs, hkv, page, d, dtype, "head", seed=3)
    table = torch.arange(2 * n_seqs, dtype=torch.int32, device="cuda").view(n_seqs, 2)
    kv = int32(INT_MIN, 20, INT_MIN + 1, 32, -1, 9, INT_MIN + rows, 1, *[12] * 8)
    zero = kv.clamp(min=0)
    for causal in (True, False):
        Q = rand((n_seqs * rows, hq * d), 9, dtype)
        news, lens = [rows] * n_seqs, [32] * n_seqs
        assert (way(ctx, Q, news, lens, hq, hkv, d, causal) if dtype == BF16 else float_way(news, lens, hq, hkv, d, causal)) == many
        starts = torch.arange(n_seqs + 1, dtype=torch.int32, device="cuda") * rows
        O, want = torch.full_like(Q, 7.0), torch.full_like(Q, 7.0)
        for lens, out in ((kv, O), (zero, want)):
            g.gelo_attention(ctx, Q, out, hq, g.KvCache(K, V), g.SeqBatch(lens, table, 32, row_start=starts, max_rows=rows), d ** -0.5, causal=causal)
        assert torch.equal(O, want) and torch.all(O.view(n_seqs, -1)[[0, 2, 4, 6]] == 0) and torch.isfinite(O.float()).all()
        # sequence 2 begins at the largest number and ends at the smallest
        starts = int32(0, 2, INT_MAX, INT_MIN, *[0] * (n_seqs - 3))
        plain = int32(0, 2, 2 + rows, *[2 + rows] * (n_seqs - 2))
        lens = torch.full_like(kv, 30)
        O, want = torch.full_like(Q, 7.0), torch.full_like(Q, 7.0)
        for at, out in ((starts, O), (plain, want)):
            g.gelo_attention(ctx, Q, out, hq, g.KvCache(K, V), g.SeqBatch(lens, table, 32, row_start=at, max_rows=rows), d ** -0.5, causal=causal)
        assert torch.equal(O, want) and torch.all(O[2 + rows:] == 7) and torch.all(O[:2 + rows] != 7)


def test_appended_rows_of_lengths_at_the_ends_of_32_bits(ctx):
    """Negative positions: zero queries, nothing appended; positions at the bound and beyond: NaN."""
    K, V = make_cache(8, 1, 16, 64, BF16, "head", fill=3.0)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(4, 2)
    batch = g.SeqBatch(int32(INT_MIN, INT_MAX, INT_MIN + 1, -1), table, 32, row_start=int32(0, 2, 4, 6, 8), max_rows=2)
    QKV, Q = rand((8, 192), 3, BF16), torch.full((8, 64), 7.0, dtype=BF16, device="cuda")
    g.gelo_rope_append(ctx, QKV, 1, g.KvCache(K, V), batch, Q=Q)
    assert torch.all(Q[[0, 1, 4, 5, 6, 7]] == 0) and torch.isnan(Q[2:4]).all()
    assert torch.all(K == 3) and torch.all(V == 3)


def test_more_rows_than_a_launch_of_the_norm_holds_are_refused(ctx):
    """Refused by their number, before anything is read: no such rows are there."""
    lib, x = g.load_library(), torch.full((64,), 5.0, device="cuda")
    p = ctypes.c_void_p(x.data_ptr())
    for n, d in ((2 ** 21 + 1, 8200), (2 ** 22, 65536), (2 ** 22 + 1, 8192)):
        status = lib.gelo_rms_norm(ctx, 0, n, d, p, d, None, 0, p, 1e-5, None, 0, p, d, None, 0, None, None)
        assert g.STATUS_NAMES[status] == "GELO_ESHAPE" and b"exceeds" in lib.gelo_last_error(ctx)
    torch.cuda.synchronize()
    assert torch.all(x == 5)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,max_rows", [(64, 2 ** 30), (64, 2 ** 30 + 16), (32, 2147418111)])
def test_a_bound_of_rows_far_above_them(ctx, dtype, hq, max_rows):
    d, page, rows = 128, 16, 100
    K, V = make_cache(8, 1, page, d, dtype, "head", seed=3)
    table, starts = torch.arange(8, dtype=torch.int32, device="cuda")[None], int32(0, rows)
    Q = rand((rows, hq * d), 9, dtype)
    O, want = torch.full_like(Q, 7.0), torch.full_like(Q, 7.0)
    for most, out in ((max_rows, O), (rows, want)):
        g.gelo_attention(ctx, Q, out, hq, g.KvCache(K, V), g.SeqBatch(int32(128), table, 128, row_start=starts, max_rows=most), d ** -0.5)
    assert torch.equal(O, want) and torch.all(O != 7)


@pytest.mark.parametrize("dtype,hq,hkv,d,new,kv,many", [(BF16, 8, 2, 64, [1, 3], [9000, 500], 0), (BF16, 8, 8, 128, [200, 30], [5000, 900], 1),
                                                        (F32, 64, 8, 96, [65, 17], [700, 300], 1), (F32, 4, 2, 128, [1, 2], [3000, 4], 0)])
def test_a_cut_cache_and_rows_of_no_sequence(ctx, dtype, hq, hkv, d, new, kv, many):
    """Rows in front of and behind those of the sequences, far more than they bring: the parts of a cut cache have no places for them, and the
    memory that was reserved is not grown."""
    front, behind, page = 300, 2000, 16
    own = g.gelo_create(0, 1)
    try:
        g.gelo_reserve_attention(own, d)
        batch, table, row_start, n_pages = make_batch(new, kv, page, 3)
        K, V = make_cache(n_pages, hkv, page, d, dtype, "head", seed=5)
        Q = rand((front + sum(new) + behind, hq * d), 8, dtype)
        O, want = torch.full_like(Q, 7.0), torch.full_like(Q, 7.0)
        inner = slice(front, front + sum(new))
        assert (way(own, Q[inner], new, kv, hq, hkv, d, True) if dtype == BF16 else float_way(new, kv, hq, hkv, d, True)) == many + 4
        padded = g.SeqBatch(batch.kv_len, batch.page_table, max(kv), row_start=torch.from_numpy(row_start).cuda() + front, max_rows=max(new))
        g.gelo_attention(own, Q[inner], want[inner], hq, g.KvCache(K, V), batch, d ** -0.5)
        torch.cuda.synchronize()
        free = torch.cuda.mem_get_info()[0]
        g.gelo_attention(own, Q, O, hq, g.KvCache(K, V), padded, d ** -0.5)
        torch.cuda.synchronize()
        assert torch.cuda.mem_get_info()[0] == free
        assert torch.equal(O, want) and torch.all(O[:front] == 7) and torch.all(O[inner.stop:] == 7) and torch.all(O[inner] != 7)
    finally:
        g.gelo_destroy(own)


LARGE_SCORES = [  # dtype, new, kv, q heads, kv heads, d, way (of float calls as float_way has it)
    (BF16, [1, 1], [200, 37], 4, 2, 64, 0), (BF16, [1, 2], [9000, 700], 4, 2, 128, 4),
    (BF16, [150] * 16, [150 + 9 * i for i in range(16)], 16, 16, 128, 1), (BF16, [150] * 16, [150 + 9 * i for i in range(16)], 16, 16, 96, 1),
    (BF16, [512, 377] * 4, [512, 400] * 4, 32, 32, 128, 2), (BF16, [200, 9], [5000, 4100], 8, 8, 64, 5), (BF16, [300], [2500], 8, 4, 256, 5),
    (F32, [1, 1], [200, 37], 4, 2, 64, 0), (F32, [1, 2], [3000, 700], 4, 2, 256, 4),
    (F32, [60] * 34, [60 + i for i in range(34)], 16, 16, 128, 1), (F32, [200, 65], [1000, 513], 16, 16, 96, 5),
]


@pytest.mark.parametrize("sign", [1, -1, 0])
@pytest.mark.parametrize("power", [20, 30, 32, 33, 40, 90])
@pytest.mark.parametrize("dtype,new,kv,hq,hkv,d,want", LARGE_SCORES)
def test_scores_that_are_large_and_finite(ctx, dtype, new, kv, hq, hkv, d, want, power, sign):
    """One component makes the scores: numbers of 8 bits, of about 2^power after the scale, exact in every type.  Different ones are at least
    2^(power - 12) apart, so a row's weights are 1 where its largest score is and 0 elsewhere: the mean of those keys' values, with a rounding of the sum
    (weights of 1 and their sum are exact) and one of the result.  sign 0: of either sign and nought, so that rows begin far below and come back."""
    page = 32
    batch, table, row_start, n_pages = make_batch(new, kv, page, 3)
    K, V = make_cache(n_pages, hkv, page, d, dtype, "head", seed=5)
    gen = torch.Generator().manual_seed(power)
    bits, shift = (torch.randint(0, n, K.shape[:3], generator=gen) for n in (128, 4))
    K.zero_()
    signs = torch.randint(-3, 2, bits.shape, generator=gen).clamp(min=-1) if sign == 0 else torch.full_like(bits, sign)
    K[..., 0] = (signs * (128 + bits) * 2.0 ** (shift - 10)).to(dtype).cuda()         # 2^-3 to 2
    Q = torch.zeros((int(row_start[-1]), hq * d), dtype=dtype, device="cuda")
    Q[:, ::d] = 2.0 ** power
    O = torch.full_like(Q, 7.0)
    assert (way(ctx, Q, new, kv, hq, hkv, d, True) if dtype == BF16 else float_way(new, kv, hq, hkv, d, True)) == want
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, 0.9)
    u = U16 if dtype == BF16 else U32
    for s in range(len(kv)):
        used = torch.from_numpy(table[s, :(kv[s] + page - 1) // page]).long().cuda()
        for h in {0, (7 * s + 5) % hq, hq - 1}:
            k, v = (x[used, h * hkv // hq].reshape(-1, d)[:kv[s]].double() for x in (K, V))
            hidden = torch.arange(kv[s], device="cuda")[None] > torch.arange(new[s], device="cuda")[:, None] + (kv[s] - new[s])
            score = k[:, 0][None].expand(new[s], -1).masked_fill(hidden, -math.inf)
            w = (score == score.amax(1, keepdim=True)).double()
            w /= w.sum(1, keepdim=True)
            got = O[int(row_start[s]):int(row_start[s + 1]), h * d:(h + 1) * d]
            within(got, host(w @ v), host(64 * U32 * (w @ v.abs()) + 1.01 * u * (w @ v).abs()), (s, h))


def refused(fn, *a, **kw):
    with pytest.raises(g.GeloError) as e:
        fn(*a, **kw)
    return g.STATUS_NAMES[e.value.status] == "GELO_EINVAL"


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 37])
def test_outputs_of_the_norm_that_share_memory(ctx, n, dtype):
    d = 264
    gamma, wide = rand((d,), 3, dtype), rand((n + 1, 4 * d), 4, dtype)
    X, R, H, out = (wide[:n, i * d:(i + 1) * d] for i in range(4))
    x, r = X.clone(), R.clone()
    want_h, want_r = torch.empty_like(x), torch.empty_like(x)
    g.gelo_rms_norm(ctx, x, gamma, 1e-6, H=want_h, residual=r, residual_out=want_r)
    # side by side in one buffer
    g.gelo_rms_norm(ctx, X, gamma, 1e-6, H=H, residual=R, residual_out=out)
    assert torch.equal(H, want_h) and torch.equal(out, want_r) and torch.equal(X, x) and torch.equal(R, r)
    before = wide.clone()
    shifted = wide.view(-1)[8:8 + n * 4 * d].view(n, 4 * d)[:, :d]                 # X, 8 values on
    bytes_of = wide.view(torch.uint8)[:n, :d]
    scales = torch.empty(n, device="cuda")
    assert refused(g.gelo_rms_norm, ctx, X, gamma, 1e-6, H=H, residual_out=H)
    assert refused(g.gelo_rms_norm, ctx, X, gamma, 1e-6, H=X, residual=R, residual_out=X)
    assert refused(g.gelo_rms_norm, ctx, X, gamma, 1e-6, H=shifted)
    assert refused(g.gelo_rms_norm, ctx, x, gamma, 1e-6, H=H, residual=X, residual_out=shifted)
    assert refused(g.gelo_rms_norm, ctx, X, gamma, 1e-6, codes=bytes_of, scales=scales)
    assert refused(g.gelo_rms_norm, ctx, x, gamma, 1e-6, H=X, codes=bytes_of, scales=scales)
    assert refused(g.gelo_rms_norm, ctx, x, gamma, 1e-6, H=H, residual_out=X, codes=bytes_of, scales=scales)
    if n > 1:                                                # of one width, but rows differently far apart
        assert refused(g.gelo_rms_norm, ctx, X, gamma, 1e-6, H=wide.view(-1)[:n * d].view(n, d))
    torch.cuda.synchronize()
    assert torch.equal(wide, before)
    g.gelo_rms_norm(ctx, X, gamma, 1e-6, H=X, residual=R, residual_out=R)          # either in the place of an input
    assert torch.equal(X, want_h) and torch.equal(R, want_r)
    X.copy_(x), R.copy_(r)
    g.gelo_rms_norm(ctx, X, gamma, 1e-6, H=R, residual=R, residual_out=X)
    assert torch.equal(R, want_h) and torch.equal(X, want_r)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 5])
def test_queries_and_results_that_share_memory(ctx, n, dtype):
    d, page = 64, 16
    K, V = make_cache(4, 1, page, d, dtype, "head", seed=3)
    cache = g.KvCache(K, V)
    batch = g.SeqBatch(int32(40), torch.arange(4, dtype=torch.int32, device="cuda")[None], 64, row_start=int32(0, n), max_rows=n)
    wide = rand((n + 1, 4 * d), 4, dtype)
    Q, O = wide[:n, :d], wide[:n, 2 * d:3 * d]
    want = torch.empty_like(Q)
    g.gelo_attention(ctx, Q.clone(), want, 1, cache, batch, 0.125)
    g.gelo_attention(ctx, Q, O, 1, cache, batch, 0.125)                            # side by side
    assert torch.equal(O, want)
    before = wide.clone()
    shifted = wide.view(-1)[8:8 + n * 4 * d].view(n, 4 * d)[:, :d]
    assert refused(g.gelo_attention, ctx, Q, Q, 1, cache, batch, 0.125) and refused(g.gelo_attention, ctx, Q, shifted, 1, cache, batch, 0.125)
    assert refused(g.gelo_attention, ctx, shifted, Q, 1, cache, batch, 0.125)
    QKV = wide[:n, :3 * d]
    keys = K.clone()
    assert refused(g.gelo_rope_append, ctx, QKV, 1, cache, batch, Q=wide[:n, d:2 * d]) and refused(g.gelo_rope_append, ctx, QKV, 1, cache, batch, Q=shifted)
    torch.cuda.synchronize()
    assert torch.equal(wide, before) and torch.equal(K, keys)
    g.gelo_rope_append(ctx, QKV, 1, cache, batch, Q=wide[:n, 3 * d:])              # behind the rows that it reads
    assert torch.equal(wide[:n, 3 * d:], before[:n, :d])
    g.gelo_rope_append(ctx, QKV, 1, cache, batch, Q=Q)
    assert torch.equal(wide[:n, :3 * d], before[:n, :3 * d])


def grid_of(codes, scales, want):
    """Codes times scales against numbers, as in the norm's test: half a step of the E4M3 grid, and 1e-6 of the grid's unit for numbers that float
    holds as multiples of 2^-149."""
    t = want / host(scales)[:, None]
    within(codes.view(torch.float8_e4m3fn), t, np.maximum(2.0 ** -4 * np.abs(t), 2.0 ** -10) + 256 * U32 * np.abs(t) + 1e-6)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [512, 4096])
def test_codes_of_rows_whose_largest_value_is_next_to_nothing(ctx, dtype, d):
    """448 over it is beyond float from 1.3e-36 down.  Every third value is nought and stays it."""
    size = torch.tensor([1e-37, 1e-38, 2e-39, 1e-39, 1e-40, 1e-41, 1.0], dtype=torch.float64)[:, None]
    x = (size * torch.randn((7, d), generator=torch.Generator().manual_seed(d), dtype=torch.float64)).to(dtype).cuda()
    x[:, ::3] = 0
    gamma = torch.ones(d, dtype=dtype, device="cuda")
    codes, scales = torch.empty((7, d), dtype=torch.uint8, device="cuda"), torch.empty(7, device="cuda")
    g.gelo_rms_norm(ctx, x, gamma, 1e-5, codes=codes, scales=scales)
    want = lo.rms_norm(host(x), host(gamma), 1e-5)[1]
    assert torch.all(codes[:, ::3] & 0x7F == 0) and torch.all(scales > 0)
    grid_of(codes, scales, want)
    if dtype == BF16:
        codes, scales = g.gelo_debug_quantize_rows_fp8(ctx, x)
        assert torch.all(codes[:, ::3] & 0x7F == 0) and torch.all(scales > 0)
        grid_of(codes, scales, host(x))


def test_codes_of_weights_whose_largest_value_is_next_to_nothing(ctx):
    """A column of the weight alike: its products are what they are with the column 2^100 times as large, over 2^100."""
    d, p = 128, 16
    U, W = rand((8, d), 3, BF16), rand((d, p), 4, BF16)
    W[::3] = 0
    Y, small = (torch.empty((8, p), dtype=BF16, device="cuda") for _ in range(2))
    W[:, 5] *= 2.0 ** -124
    g.gelo_project_fp8(ctx, U, g.gelo_prepare_weight_fp8(ctx, W), p, small)
    W[:, 5] *= 2.0 ** 100
    g.gelo_project_fp8(ctx, U, g.gelo_prepare_weight_fp8(ctx, W), p, Y)
    rest = [c for c in range(p) if c != 5]
    assert torch.equal(Y[:, rest], small[:, rest])
    got, want = host(small[:, 5]), host(U) @ host(W[:, 5]) * 2.0 ** -100
    assert np.linalg.norm(got - want) < 2 * 2.0 ** -4 * np.linalg.norm(want)


WHOLE_WEIGHTS = [  # new, kv, q heads, kv heads, d, way
    ([1] * 5, [200, 3, 77, 130, 256], 4, 2, 64, 0), ([1] * 3, [2100, 900, 17], 8, 8, 96, 4), ([1] * 2, [513, 1030], 48, 2, 128, 4),
    ([1] * 3, [77, 250, 129], 16, 2, 256, 0), ([3, 20, 11], [70, 200, 256], 3, 3, 128, 0), ([2], [1500], 8, 1, 256, 4),
]


@pytest.mark.parametrize("new,kv,hq,hkv,d,want", WHOLE_WEIGHTS)
def test_few_columns_keep_their_weights(ctx, new, kv, hq, hkv, d, want):
    """bfloat16 with few columns: a weight is the sum of two bfloat16, off by half a unit of the second, at most 2^-7 of the first: 2^-16 of the
    weight.  With it the float bounds of the other tests and one rounding of the result, for which nothing is allowed but U16 of itself: values that
    cancel in the sum must not be moved by what rounding the weights to 8 bits would move them."""
    page = 16
    batch, table, row_start, n_pages = make_batch(new, kv, page, 3)
    K, V = make_cache(n_pages, hkv, page, d, BF16, "head", seed=5)
    Q = rand((int(row_start[-1]), hq * d), 8, BF16)
    O = torch.full_like(Q, 7.0)
    assert way(ctx, Q, new, kv, hq, hkv, d, True) == want
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, d ** -0.5)
    ref, absolute = lo.attention(host(Q), host(K), host(V), hq, row_start, kv, table, d ** -0.5, True)
    bound = attention_bound(ref, absolute, host(Q), host(K), d ** -0.5, max(kv), d, F32) + 2.0 ** -16 * absolute + 1.01 * U16 * np.abs(ref)
    within(O, ref, bound)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d", [(1, 2056), (3, 4096), (65, 4088), (65, 4096), (7, 3000)])
def test_norm_without_codes(ctx, n, d, dtype):
    """The widths at which a row has more threads where no codes are asked for.  Bounds as in test_norm."""
    x, r, gamma = rand((n, d), d, dtype, 3.0), rand((n, d), d + 1, dtype), rand((d,), d + 2, dtype)
    u = U16 if dtype == BF16 else 0.0
    for residual in (None, r):
        for keep in (False, True):
            H, H_all = base.padded(n, d, d + 8, dtype)
            R, R_all = base.padded(n, d, d + 16, dtype)
            g.gelo_rms_norm(ctx, x, gamma, 1e-5, H=H, residual=residual, residual_out=R if keep else None)
            h, y = lo.rms_norm(host(x), host(gamma), 1e-5, None if residual is None else host(residual))
            within(H, y, (64 * U32 + u) * np.abs(y) * 1.01 + 1e-38, "H")
            assert torch.all(H_all[:, d:] == 7) and torch.all(R_all[:, d if keep else 0:] == 7)
            if keep:
                within(R, h, (U32 + u) * np.abs(h) * 1.01, "residual")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [512, 2048, 4096, 8192, 16384, 65536])
def test_norms_whose_results_are_stored_past_the_caches(ctx, d, dtype):
    """More than 40 MB of results, for every number of threads to a row; in float64 on the GPU, bounds as in test_norm."""
    size = 2 if dtype == BF16 else 4
    n = 21_000_000 // (d * size) + 3
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, r = ((3 * torch.randn((n, d), generator=gen, device="cuda")).to(dtype) for _ in range(2))
    gamma = torch.randn(d, generator=gen, device="cuda").to(dtype)
    H, R = (torch.full((n, d + 8), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    assert 2 * n * d * size > 40e6
    g.gelo_rms_norm(ctx, x, gamma, 1e-5, H=H[:, :d], residual=r, residual_out=R[:, :d])
    h = x.double() + r.double()
    y = h / (h.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * gamma.double()
    u = U16 if dtype == BF16 else 0.0
    assert torch.all((R[:, :d].double() - h).abs() <= (U32 + u) * 1.01 * h.abs())
    assert torch.all((H[:, :d].double() - y).abs() <= (64 * U32 + u) * 1.01 * y.abs() + 1e-38)
    assert torch.all(H[:, d:] == 7) and torch.all(R[:, d:] == 7)


LARGE_CACHES = [  # dtype, sequences, kv (fewest, most), q heads, kv heads, d, page
    (BF16, 64, (350, 512), 16, 8, 128, 16), (BF16, 64, (100, 128), 32, 32, 128, 64), (BF16, 64, (40, 64), 64, 32, 256, 16), (BF16, 32, (300, 512), 16, 8, 256, 32),
    (BF16, 64, (200, 256), 32, 32, 64, 32), (F32, 64, (40, 64), 32, 32, 128, 16), (F32, 64, (30, 64), 32, 32, 256, 16), (BF16, 3, (20000, 32767), 32, 8, 128, 64),
]


@pytest.mark.parametrize("order", ["head", "row"])
@pytest.mark.parametrize("dtype,n_seqs,lengths,hq,hkv,d,page", LARGE_CACHES)
def test_single_tokens_against_caches_that_are_read_past_the_caches(ctx, dtype, n_seqs, lengths, hq, hkv, d, page, order):
    """More than 100 MB of keys and values; where the heads of a row lie side by side and are 2048 and more in all, a wave has a head.  The
    reference in float64 on the GPU, for every sequence and three of the heads."""
    rng = np.random.default_rng(d)
    kv = [lengths[1]] + [int(x) for x in rng.integers(lengths[0], lengths[1] + 1, n_seqs - 1)]
    batch, table, row_start, n_pages = make_batch([1] * n_seqs, kv, page, 3, one_row=True)
    gen = torch.Generator(device="cuda").manual_seed(d)
    shape = (n_pages, hkv, page, d) if order == "head" else (n_pages, page, hkv, d)
    K, V = (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype) for _ in range(2))
    if order == "row":
        K, V = K.permute(0, 2, 1, 3), V.permute(0, 2, 1, 3)
    assert 2 * K.element_size() * n_seqs * hkv * max(kv) * d > 100e6
    Q, O = rand((n_seqs, hq * d), 8, dtype), torch.full((n_seqs, hq * d), 7.0, dtype=dtype, device="cuda")
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), batch, d ** -0.5)
    assert torch.isfinite(O.float()).all()
    for s in range(n_seqs):
        used = torch.from_numpy(table[s, :(kv[s] + page - 1) // page]).long().cuda()
        for h in {0, (7 * s + 5) % hq, hq - 1}:
            k, v = (x[used, h * hkv // hq].reshape(-1, d)[:kv[s]].double() for x in (K, V))
            q = Q[s:s + 1, h * d:(h + 1) * d].double()
            w = torch.softmax(q @ k.T * d ** -0.5, -1)
            ref, absolute = host(w @ v), host(w @ v.abs())
            within(O[s:s + 1, h * d:(h + 1) * d], ref, attention_bound(ref, absolute, host(q), host(k), d ** -0.5, kv[s], d, dtype), (s, h))


@pytest.mark.parametrize("new,kv,hq,d,want", [([60] * 34 + [3], [60] * 34 + [0], 16, 128, 1), ([60] * 34 + [3], [60] * 34 + [0], 16, 96, 1),
                                              ([200, 65, 4], [1000, 513, 0], 16, 96, 5), ([200, 65, 4], [1000, 513, 0], 16, 128, 5)])
def test_float_by_tiles_of_64_columns_and_a_row_without_a_softmax(ctx, new, kv, hq, d, want):
    """Float has two kernels: the one for tiles of 64 columns, the cache whole and cut."""
    assert float_way(new, kv, hq, hq, d, True) == want
    base.test_a_row_that_sees_only_scores_of_minus_infinity_has_no_softmax(ctx, F32, new, kv, hq, d, None)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 96)])
@pytest.mark.parametrize("n_seqs,rows", [(1, 1), (2, 40), (40, 20)])
def test_a_bound_of_lengths_near_2_to_the_31(ctx, dtype, d, n_seqs, rows):
    """A captured launch may be sized for any length; pages of 65536 rows keep the table short."""
    hq, page, most = 16, 65536, 2 ** 31 - 65537
    K, V = make_cache(2, hq, page, d, dtype, "row", seed=3)
    table = torch.zeros((n_seqs, 32768), dtype=torch.int32, device="cuda")
    table[:, 0] = 1
    kv = torch.arange(200, 200 + n_seqs, dtype=torch.int32, device="cuda")
    starts = torch.arange(n_seqs + 1, dtype=torch.int32, device="cuda") * rows
    Q = rand((n_seqs * rows, hq * d), 9, dtype)
    O = torch.full_like(Q, 7.0)
    g.gelo_attention(ctx, Q, O, hq, g.KvCache(K, V), g.SeqBatch(kv, table, most, row_start=starts, max_rows=rows), d ** -0.5)
    for h in (0, hq - 1):
        at = slice(h * d, (h + 1) * d)
        ref, absolute = lo.attention(host(Q[:, at]), host(K[:, h:h + 1, :256]), host(V[:, h:h + 1, :256]), 1, starts.tolist(), kv.tolist(), table.cpu().numpy(), d ** -0.5, True)
        within(O[:, at], ref, attention_bound(ref, absolute, host(Q), host(K[:, :, :256]), d ** -0.5, 256, d, dtype), h)
