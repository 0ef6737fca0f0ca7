"""Low-rank adapters beside a projection, through the C ABI, against the float64 reference.

Bounds, element by element, from the formats' unit roundoffs U32 = 2^-24 and U16 = 2^-8 (bfloat16); see adapt_bound."""
import ctypes

import numpy as np
import pytest
import torch

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


def adapt_bound(Z, size, d, rank, dtype):
    """`size`: |base| + sum of the sizes of all terms.  The inner sum errs by (d + 20) U32 of its terms' sizes, the outer one by (rank + 20) U32, its factor by one.
    bfloat16: the inner sum is two bfloat16, the first 8 bits of it and the rest, below 2^-7 of it, rounded at 2^-8 of itself: 2^-15.  One rounding at the end."""
    e = U32 * (d + rank + 45)
    if dtype == BF16:
        return 1.01 * ((e + 2.0 ** -15) * size + U16 * np.abs(Z)) + 1e-30
    return 1.01 * (e * size + U32 * np.abs(Z)) + 1e-30


def make(n, d, parts, rank, count, dtype, seed, gap=0):
    """H, base, A, B with leading dimensions `gap` values wider than their rows, scale, part ends."""
    ends = list(np.cumsum(parts))
    p = int(ends[-1])
    H, _ = padded(n, d, d + gap, dtype)
    base, _ = padded(n, p, p + gap, dtype)
    H.copy_(rand((n, d), seed, dtype, 2.0))
    base.copy_(rand((n, p), seed + 1, dtype))
    A = torch.full((count, len(parts) * rank + gap // 8, d + gap), 9.0, dtype=dtype, device="cuda")[:, :len(parts) * rank, :d]
    B = torch.full((count, p + gap // 8, rank + gap), 9.0, dtype=dtype, device="cuda")[:, :p, :rank]
    A.copy_(rand(A.shape, seed + 2, dtype, d ** -0.5))
    B.copy_(rand(B.shape, seed + 3, dtype, 0.3))
    scale = (0.5 + torch.rand(count, generator=torch.Generator().manual_seed(seed + 4))).cuda()
    return H, base, A, B, scale, [int(e) for e in ends]


def check(ctx, H, base, A, B, scale, ends, which, dtype, rows=None):
    n, p = base.shape
    d, rank = H.shape[1], B.shape[2]
    Z, Z_all = padded(n, p, p + 24, dtype)
    ids = torch.tensor(which, dtype=torch.int32).cuda()
    adapters = g.Adapters(A, B, scale=scale, part_ends=ends)
    kept = base.clone()
    g.gelo_adapt(ctx, H, adapters, ids, Z, base=base)
    assert torch.all(Z_all[:, p:] == 7) and torch.equal(base, kept)
    rows = np.arange(n) if rows is None else np.asarray(rows)
    s = [1.0] * A.shape[0] if scale is None else host(scale)
    want, size = so.adapt(host(H)[rows], host(base)[rows], host(A), host(B), s, [which[i] for i in rows], ends)
    off = np.abs(host(Z)[rows] - want) - adapt_bound(want, size, d, rank, dtype)
    assert off.max() <= 0, (float(off.max()), np.unravel_index(off.argmax(), off.shape))
    none = torch.tensor([not 0 <= w < A.shape[0] for w in which]).cuda()
    assert torch.equal(Z[none], base[none])
    in_place = base.clone()
    g.gelo_adapt(ctx, H, adapters, ids, in_place)
    assert torch.equal(in_place, Z)
    return Z


def way(n, d, p, rank, parts, count, dtype):
    """0: rows by themselves, 1: groups of rows as they come, 2: groups of rows put in order."""
    return ctypes.CDLL(g.LIB_PATH)["_ZN4gelo9adapt_wayEiiiiiii"](int(dtype == BF16), n, d, p, rank, parts, count)


CASES = [  # n, d, widths of the parts, rank, adapters
    (1, 8, (8,), 8, 1),
    (3, 72, (16, 24), 8, 2),
    (17, 264, (64, 16, 48), 16, 5),
    (64, 1024, (256, 64, 64), 16, 48),
    (65, 200, (144,), 24, 7),
    (16, 4096, (512,), 64, 16),
    (40, 1000, (16, 16, 16, 8), 128, 3),
    (300, 96, (80, 40), 40, 30),
    (130, 520, (1040,), 56, 1),
    (700, 64, (72,), 8, 600),
    (1025, 136, (96, 32, 32), 16, 9),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gap", [0, 16])
@pytest.mark.parametrize("n,d,parts,rank,count", CASES)
def test_adapters_in_any_order(ctx, n, d, parts, rank, count, gap, dtype):
    rng = np.random.default_rng(n)
    which = [int(w) for w in rng.integers(-1, count + 1, n)]                     # -1 and `count`: none
    check(ctx, *make(n, d, parts, rank, count, dtype, n + d, gap), which, dtype)


GROUPS = [  # n, d, widths of the parts, rank, adapters, way
    (300, 1032, (1040,), 128, 1, 1),
    (513, 1000, (560, 48, 24), 72, 2, 1),
    (1000, 520, (272, 512), 104, 4, 1),
    (4100, 1024, (1264,), 8, 3, 1),
    (700, 1000, (512, 256, 248), 40, 600, 2),
    (1025, 1544, (1024, 16), 24, 9, 2),
    (2050, 800, (800,), 56, 30, 2),
    (1100, 1000, (1000,), 128, 5, 2),
    (2100, 1000, (1000,), 32, 8, 1),
    (5000, 2048, (256, 256, 256), 16, 1200, 2),
    (9000, 1024, (1024,), 8, 70, 2),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("order", ["any", "runs", "one"])
@pytest.mark.parametrize("n,d,parts,rank,count,want", GROUPS)
def test_groups_of_rows(ctx, n, d, parts, rank, count, want, order, dtype):
    """Rows in any order, side by side (prompts: runs whose ends lie inside tiles), and all but a few of one adapter; some without one.  A row of each tile and all that are
    next to a change are looked at."""
    assert way(n, d, sum(parts), rank, len(parts), count, dtype) == want
    rng = np.random.default_rng(n)
    which = [int(w) for w in rng.integers(-1, count + 1, n)] if order == "any" else [i * count // n for i in range(n)] if order == "runs" else [count - 1] * n
    for i in (range(100, 137) if order != "any" else []):
        which[i] = -1
    if order == "one":
        which[5] = which[n - 1] = 0
    rows = sorted({i for i in range(0, n, 61)} | {i for i in range(1, n) if order != "any" and which[i] != which[i - 1]} | {n - 1})[:150] + [n - 1]
    check(ctx, *make(n, d, parts, rank, count, dtype, n + d, 8), which, dtype, rows=rows)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("count,want", [(3, 1), (20, 2)])
@pytest.mark.parametrize("n", [319, 320, 321, 335, 336, 337, 351, 352, 353, 383, 384, 385])
def test_numbers_of_rows_at_the_edges_of_groups(ctx, n, count, want, dtype):
    """The last group is of 63, 64, 1 ... rows."""
    assert way(n, 1400, 800, 128, 1, count, dtype) == want
    check(ctx, *make(n, 1400, (800,), 128, count, dtype, n, 8), [(i // 5) % (count + 1) - 1 for i in range(n)], dtype, rows=[*range(0, n, 40), *range(n - 20, n)])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 271, 272, 273])
def test_numbers_of_rows_at_the_edges_of_tiles(ctx, n, dtype):
    check(ctx, *make(n, 104, (64, 72), 8, 3, dtype, n, 8), [(i // 5) % 4 - 1 for i in range(n)], dtype)


WHOLE = [  # n, d, widths of the parts, rank, adapters, launches in bfloat16 and float
    (5, 1024, (1032,), 8, 3, (1, 1)), (5, 1032, (528, 16, 8), 24, 3, (1, 2)), (7, 2048, (48, 32), 16, 2, (1, 2)), (7, 2056, (48, 32), 16, 2, (2, 2)), (33, 40, (1536,), 32, 9, (1, 1)), (3, 1024, (64, 512), 32, 2, (1, 2)),
    (9, 8, (16, 24), 32, 3, (1, 1)), (9, 8, (16, 24), 40, 3, (2, 2)), (500, 512, (512, 512, 512), 16, 64, (1, 2)), (700, 72, (528,), 8, 700, (1, 1))]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gap", [0, 16])
@pytest.mark.parametrize("n,d,parts,rank,count,launches", WHOLE)
def test_small_rows_in_one_launch(ctx, n, d, parts, rank, count, launches, gap, dtype):
    go = ctypes.CDLL(g.LIB_PATH)["_ZN4gelo14adapt_launchesEiiiiiii"]
    assert go(int(dtype == BF16), n, d, sum(parts), rank, len(parts), count) == launches[dtype == F32]
    H, base, A, B, scale, ends = make(n, d, parts, rank, count, dtype, 17, gap)
    ids = np.random.default_rng(4).integers(-1, count + 1, n)
    check(ctx, H, base, A, B, scale, ends, [int(x) for x in ids], dtype)
    check(ctx, H, base, A, B, None, ends, [0] * n, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d,rank,count", [(1, 136, 16, 4), (20, 136, 16, 4), (600, 1400, 104, 4), (600, 1400, 104, 9)])
def test_without_factors_and_without_any_adapter(ctx, n, d, rank, count, dtype):
    H, base, A, B, _, ends = make(n, d, (48, 16), rank, count, dtype, n)
    rows = range(0, n, max(1, n // 50))
    check(ctx, H, base, A, B, None, ends, [i % count for i in range(n)], dtype, rows)
    Z = check(ctx, H, base, A, B, None, ends, [-(2 ** 31) if i % 2 else 2 ** 31 - 1 for i in range(n)], dtype, rows)
    assert torch.equal(Z, base)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d,rank,count,want", [(40, 136, 16, 4, 0), (700, 1400, 48, 4, 1), (700, 1400, 64, 9, 2)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_finite_reaches_only_its_rows(ctx, bad, n, d, rank, count, want, dtype):
    """In one row of H, in A and in B of one adapter, in base: everything else keeps its bits.  An infinity in B's column: that column."""
    H, base, A, B, scale, ends = make(n, d, (48, 32), rank, count, dtype, 3)
    assert way(n, d, 80, rank, 2, count, dtype) == want
    which = [i % 5 - 1 for i in range(n)]
    ids = torch.tensor(which, dtype=torch.int32).cuda()

    def run(H=H, base=base, A=A, B=B):
        Z = torch.empty_like(base)
        return g.gelo_adapt(ctx, H, g.Adapters(A, B, scale=scale, part_ends=ends), ids, Z, base=base)
    clean = run()
    assert torch.isfinite(clean.float()).all()
    h = H.clone()
    h[7, 100] = bad
    h[10, 3] = bad                                           # without an adapter
    Z = run(H=h)
    rest = torch.ones(n, dtype=torch.bool)
    rest[7] = False
    assert which[7] >= 0 and which[10] == -1
    assert torch.equal(Z[rest], clean[rest]) and not torch.isfinite(Z[7].float()).any()
    for name, m, where in (("A", A, (2, rank + 1, 5)), ("B", B, (2, 50, 3))):
        x = m.clone()
        x[where] = bad
        Z = run(**{name: x})
        mine = ids == 2
        assert torch.equal(Z[~mine], clean[~mine])
        cols = torch.zeros(80, dtype=torch.bool)
        cols[48 if name == "A" else 50:80 if name == "A" else 51] = True         # that row of A is the second part's
        assert not torch.isfinite(Z[mine][:, cols].float()).any() and torch.equal(Z[mine][:, ~cols], clean[mine][:, ~cols])
    b = base.clone()
    b[9, 11] = bad
    Z = run(base=b)
    same = torch.ones_like(Z, dtype=torch.bool)
    same[9, 11] = False
    assert torch.equal(Z[same], clean[same]) and not torch.isfinite(Z[9, 11].float())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d,rank,count,want", [(40, 136, 16, 4, 0), (900, 1400, 16, 4, 1), (700, 1400, 48, 4, 1), (700, 1400, 64, 9, 2)])
def test_an_infinite_weight_has_the_sign_of_what_it_meets(ctx, n, d, rank, count, want, dtype):
    """T whole numbers of few bits, which a bfloat16 holds with nothing left: T times an infinity is one."""
    parts, p = (48, 32), 80
    H, base, A, B, scale, ends = make(n, d, parts, rank, count, dtype, 3)
    H.copy_(torch.randint(1, 3, H.shape, generator=torch.Generator().manual_seed(1)))
    A.zero_()
    A[:, :, 0] = 1.0
    A[:, 3, 0] = -1.0                                        # of the first part's ranks
    assert way(n, d, p, rank, 2, count, dtype) == want
    B[1, 5, 3] = float("inf")
    B[1, 6, 2] = float("inf")
    B[1, 60, 3] = float("-inf")
    ids = torch.tensor([i % count for i in range(n)], dtype=torch.int32).cuda()
    Z = g.gelo_adapt(ctx, H, g.Adapters(A, B, part_ends=ends), ids, torch.empty_like(base), base=base)
    mine = Z[ids == 1].float()
    assert (mine[:, [5, 60]] == -float("inf")).all() and (mine[:, 6] == float("inf")).all()
    mine[:, [5, 6, 60]] = 0
    assert torch.isfinite(mine).all() and torch.isfinite(Z[ids != 1].float()).all()


FACTORS = [(9, 64, 8, 4, 0), (40, 136, 64, 4, 0), (700, 1400, 48, 4, 1), (700, 1400, 64, 9, 2)]          # n, d, rank, adapters, way


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d,rank,count,want", FACTORS)
@pytest.mark.parametrize("inner,outer,factor", [(1e12, 1e-30, 1e27), (1e-20, 1e28, 1e-25)])
def test_factors_that_the_inner_sum_could_not_take(ctx, inner, outer, factor, n, d, rank, count, want, dtype):
    """A factor multiplies the sum over the ranks: inner sums of 1e12 times 1e27 leave float's range upwards, of 1e-20 times 1e-25 downwards, the sums of their products with B and what
    these are times the factor (1e9, 1e-17) stay far inside."""
    H, base, A, B, scale, ends = make(n, d, (48, 32), rank, count, dtype, 11)
    assert way(n, d, 80, rank, 2, count, dtype) == want
    A.mul_(inner), B.mul_(outer), scale.mul_(factor)
    if factor < 1:
        base.zero_()
    check(ctx, H, base, A, B, scale, ends, [i % (count + 1) - 1 for i in range(n)], dtype, range(0, n, max(1, n // 60)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d,rank,count,want", FACTORS)
def test_an_infinite_factor_has_the_sign_of_the_sum(ctx, n, d, rank, count, want, dtype):
    """Sums that are off from 0 by more than they can err; everything else keeps its bits."""
    H, base, A, B, scale, ends = make(n, d, (48, 32), rank, count, dtype, 12)
    assert way(n, d, 80, rank, 2, count, dtype) == want
    which = [i % (count + 1) - 1 for i in range(n)]
    ids = torch.tensor(which, dtype=torch.int32).cuda()
    clean = g.gelo_adapt(ctx, H, g.Adapters(A, B, scale=scale, part_ends=ends), ids, torch.empty_like(base), base=base)
    odd = scale.clone()
    odd[1] = float("inf")
    Z = g.gelo_adapt(ctx, H, g.Adapters(A, B, scale=odd, part_ends=ends), ids, torch.empty_like(base), base=base)
    mine = ids == 1
    assert torch.equal(Z[~mine], clean[~mine])
    rows = [i for i in range(n) if which[i] == 1][:60]
    added, size = so.adapt(host(H)[rows], 0 * host(base)[rows], host(A), host(B), [1.0] * count, [1] * len(rows), ends)
    sure = np.abs(added) > adapt_bound(0 * added, size, d, rank, dtype)
    assert sure.mean() > 0.9 and np.array_equal(host(Z)[rows][sure], np.sign(added[sure]) * np.inf)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d,rank,count,want", [(33, 264, 16, 6, 0), (600, 1400, 56, 4, 1), (600, 1400, 80, 6, 2)])
def test_a_row_s_bits_do_not_go_by_the_rows_around_it(ctx, n, d, rank, count, want, dtype):
    """The same rows in another order, and with other adapters beside them."""
    H, base, A, B, scale, ends = make(n, d, (48, 32), rank, count, dtype, 5)
    assert way(n, d, 80, rank, 2, count, dtype) == want
    adapters = g.Adapters(A, B, scale=scale, part_ends=ends)
    which = torch.randint(0, count, (n,), generator=torch.Generator().manual_seed(1)).int().cuda()
    Z, Y = torch.empty_like(base), torch.empty_like(base)
    g.gelo_adapt(ctx, H, adapters, which, Z, base=base)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(2)).cuda()
    g.gelo_adapt(ctx, H[order].contiguous(), adapters, which[order].contiguous(), Y, base=base[order].contiguous())
    assert torch.equal(Y, Z[order])
    g.gelo_adapt(ctx, H, adapters, which, Y, base=base)
    assert torch.equal(Y, Z)


def test_one_a_for_all_adapters(ctx):
    """A stride of 0."""
    H, base, A, B, scale, ends = make(50, 136, (48, 32), 16, 4, BF16, 5)
    check(ctx, H, base, A[:1].expand(4, -1, -1), B, scale, ends, [i % 4 for i in range(50)], BF16)


@pytest.mark.parametrize("n,ways", [(16, (0, 0)), (70, (2, 1))])
def test_adapters_beyond_32_bit_offsets(ctx, n, ways):
    """Adapters 2^31 values and more behind the first one's."""
    count, rank, d, p = 1100, 128, 8192, 8192
    assert (way(n, d, p, rank, 1, count, BF16), way(n, d, p, rank, 1, 1, BF16)) == ways
    A, B = (torch.zeros((count, *s), dtype=BF16, device="cuda") for s in ((rank, d), (p, rank)))
    last = count - 1
    A[last], B[last] = rand((rank, d), 1, BF16, d ** -0.5), rand((p, rank), 2, BF16, 0.3)
    H, base = rand((n, d), 3, BF16), rand((n, p), 4, BF16)
    Z, want = torch.empty_like(base), torch.empty_like(base)
    g.gelo_adapt(ctx, H, g.Adapters(A, B), torch.full((n,), last, dtype=torch.int32).cuda(), Z, base=base)
    g.gelo_adapt(ctx, H, g.Adapters(A[last:], B[last:]), torch.zeros(n, dtype=torch.int32).cuda(), want, base=base)
    assert torch.equal(Z, want) and not torch.equal(Z, base)


def test_workspace_that_is_outgrown_serves_captured_calls(ctx):
    """A captured call keeps its workspace's address: a larger call later takes another one."""
    c = g.gelo_create(0, 1)
    try:
        H, base, A, B, scale, ends = make(20, 2056, (48, 32), 16, 4, BF16, 5)
        adapters = g.Adapters(A, B, scale=scale, part_ends=ends)
        which = torch.tensor([i % 4 for i in range(20)], dtype=torch.int32).cuda()
        Z, Y = torch.empty_like(base), torch.empty_like(base)
        go = ctypes.CDLL(g.LIB_PATH)["_ZN4gelo14adapt_launchesEiiiiiii"]
        assert go(1, 20, 2056, 80, 16, 2, 4) == 2            # (a call in one launch has no use for it)
        g.gelo_reserve_adapt(c, 20, 16, 2, 4)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            g.gelo_adapt(c, H, adapters, which, Z, base=base)
        big = make(3000, 1400, (48, 32), 16, 4, BF16, 6)
        for turn in range(3):
            H.copy_(rand(H.shape, 30 + turn, BF16))
            graph.replay()
            check(c, *big[:5], big[5], [i % 4 for i in range(3000)], BF16, rows=range(0, 3000, 97))
            torch.cuda.synchronize()
            got = Z.clone()
            g.gelo_adapt(ctx, H, adapters, which, Y, base=base)
            assert torch.equal(got, Y)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(Z, Y)
    finally:
        g.gelo_destroy(c)


def test_behind_the_obfuscated_projection(ctx):
    """Beside gelo_qkv_forward: Z of the protocol, then what the adapters add to it, in place; against the plain product with the merged weight.  The projection may be
    off by its contract, 2e-2 of |H W| in the Frobenius norm, the addition by far less."""
    n, d, p, rank = 48, 512, 384, 16
    c = g.gelo_create(0, 77)
    try:
        H, W = rand((n, d), 1, BF16), rand((d, p), 2, BF16, d ** -0.5)
        A, B = rand((2, rank, d), 3, BF16, d ** -0.5), rand((2, p, rank), 4, BF16, 0.3)
        Z = torch.empty((n, p), dtype=BF16, device="cuda")
        g.gelo_qkv_forward(c, g.GELO_ORTHOGONAL, H, W, Z, k_shield=4, batch_id=0)
        which = torch.tensor([i % 3 for i in range(n)], dtype=torch.int32).cuda()          # 2: none
        g.gelo_adapt(c, H, g.Adapters(A, B), which, Z)
        want = host(H) @ host(W)
        plain = np.linalg.norm(want)
        for i in range(n):
            if i % 3 < 2:
                want[i] += host(B[i % 3]) @ (host(A[i % 3]) @ host(H[i]))
        assert np.linalg.norm(host(Z) - want) < 2e-2 * plain + 2 * U16 * np.linalg.norm(want)
    finally:
        g.gelo_destroy(c)


def test_refusals(ctx):
    lib, P = g.load_library(), ctypes.c_void_p
    buf = torch.full((1 << 16,), 5.0, device="cuda")
    ints = torch.zeros(64, dtype=torch.int32, device="cuda")
    x, i = buf.data_ptr(), ints.data_ptr()

    def call(dtype=0, n=4, d=64, p=80, H=x, ldh=64, which=i, base=x + 8192, ldb=80, Z=x + 16384, ldz=80, **kw):
        a = dict(a=x, b=x, scale=x, n_adapters=3, rank=8, n_parts=2, part_end=(32, 80), a_stride=1024, lda=64, b_stride=640, ldb=8)
        a.update({k.replace("b_ldb", "ldb"): v for k, v in kw.items()})
        a["part_end"] = (ctypes.c_int * 4)(*a["part_end"])
        s = g._AdaptersStruct(*a.values())
        return g.STATUS_NAMES[lib.gelo_adapt(ctx, dtype, n, d, p, P(H), ldh, ctypes.byref(s), P(which), P(base), ldb, P(Z), ldz, P(None))]
    for bad in ({"dtype": 2}, {"n": 0}, {"d": 0}, {"p": 0}, {"H": None}, {"base": None}, {"Z": None}, {"which": None}, {"a": None}, {"b": None}, {"n_adapters": 0},
                {"rank": 0}, {"n_parts": 0}, {"part_end": (32, 72)}, {"part_end": (24, 80)}, {"part_end": (80, 80)}, {"part_end": (0, 80)}, {"ldh": 56}, {"ldb": 72}, {"ldz": 72},
                {"lda": 56}, {"b_ldb": 0}, {"Z": x}, {"Z": x + 8192 + 160}, {"Z": x + 8192, "ldz": 88}):
        assert call(**bad) == "GELO_EINVAL", bad
    for bad in ({"rank": 12}, {"rank": 136, "b_ldb": 136}, {"n_parts": 5}, {"a_stride": -8}, {"lda": (1 << 24) + 8}, {"b_ldb": (1 << 24) + 8}):
        assert call(**bad) == "GELO_ESHAPE", bad
    for bad in ({"d": 60}, {"p": 76, "part_end": (32, 76)}, {"H": x + 4}, {"Z": x + 16388}, {"ldh": 68}, {"a": x + 8}, {"lda": 68}, {"a_stride": 1028}, {"b_stride": 644},
                {"which": i + 2}, {"scale": x + 1}):
        assert call(**bad) == "GELO_EALIGN", bad
    st = lib.gelo_adapt(ctx, 0, 4, 64, 80, P(x), 64, None, P(i), P(x + 8192), 80, P(x + 16384), 80, P(None))
    assert g.STATUS_NAMES[st] == "GELO_EINVAL"
    for bad, want in (((0, 8, 1, 1), "GELO_EINVAL"), ((4, 8, 1, 0), "GELO_EINVAL"), ((4, 12, 1, 1), "GELO_ESHAPE"), ((4, 8, 5, 1), "GELO_ESHAPE"),
                      ((4, 136, 1, 1), "GELO_ESHAPE")):
        with pytest.raises(g.GeloError) as e:
            g.gelo_reserve_adapt(ctx, *bad)
        assert g.STATUS_NAMES[e.value.status] == want, bad
    torch.cuda.synchronize()
    assert torch.all(buf == 5)
