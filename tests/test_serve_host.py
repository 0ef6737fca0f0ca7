"""The host's side of the cache of 4 bits and of adapters: what the binding makes of tensors and refuses, and what the library reckons from sizes.  Nothing
here launches a kernel or needs a GPU."""
import ctypes
import random

import pytest
import torch

from paper_2603_05035_amd import binding as g


class OnGpu(torch.Tensor):
    """A host tensor that says it lives on the GPU: for code that looks at shapes and strides only."""

    @property
    def is_cuda(self):
        return True


def on_gpu(t):
    return t.as_subclass(OnGpu)


def zeros(*shape, dtype=torch.bfloat16):
    return on_gpu(torch.zeros(shape, dtype=dtype))


def test_bytes_of_a_piece():
    lib = g.load_library()
    for page, d in ((16, 32), (16, 64), (64, 96), (128, 128), (16, 256), (1 << 20, 256)):
        assert g.gelo_fp4_page_bytes(page, d) == page * d * 17 // 32
    v = ctypes.c_size_t(5)
    for page, d, want in ((0, 64, "GELO_EINVAL"), (16, 0, "GELO_EINVAL"), (8, 64, "GELO_ESHAPE"), (48, 64, "GELO_ESHAPE"), (16, 48, "GELO_ESHAPE"),
                          (1 << 24, 32, "GELO_ESHAPE")):
        assert g.STATUS_NAMES[lib.gelo_fp4_page_bytes(page, d, ctypes.byref(v))] == want, (page, d)
    assert v.value == 5 and g.STATUS_NAMES[lib.gelo_fp4_page_bytes(16, 64, None)] == "GELO_EINVAL"
    with pytest.raises(g.GeloError):
        g.gelo_fp4_page_bytes(24, 64)


def test_a_cache_s_strides_are_those_of_its_tensors():
    piece = g.gelo_fp4_page_bytes(16, 64)
    s = g.KvCacheFp4(zeros(5, 3, piece, dtype=torch.uint8), zeros(5, 3, piece, dtype=torch.uint8), 16, 64).struct
    assert (s.n_pages, s.n_kv_heads, s.page_rows, s.head_dim, s.page_stride, s.head_stride) == (5, 3, 16, 64, 3 * piece, piece)
    both = zeros(5, 2, 3, piece + 16, dtype=torch.uint8)
    s = g.KvCacheFp4(both[:, 0, :, :piece], both[:, 1, :, :piece], 16, 64).struct
    assert (s.page_stride, s.head_stride) == (6 * (piece + 16), piece + 16)
    heads_first = zeros(3, 5, piece, dtype=torch.uint8).permute(1, 0, 2)
    s = g.KvCacheFp4(heads_first, heads_first, 16, 64).struct
    assert (s.page_stride, s.head_stride) == (piece, 5 * piece)
    one = zeros(1, 1, piece, dtype=torch.uint8)
    assert g.KvCacheFp4(one, one, 16, 64).struct.head_stride % 16 == 0


def test_caches_that_are_refused():
    piece = g.gelo_fp4_page_bytes(16, 64)
    good = zeros(5, 3, piece, dtype=torch.uint8)
    for K, V in ((good, zeros(5, 3, piece)), (good, zeros(4, 3, piece, dtype=torch.uint8)), (good[..., :-1], good[..., :-1]), (torch.zeros_like(good).as_subclass(torch.Tensor), good),
                 (good, zeros(3, 5, piece, dtype=torch.uint8).permute(1, 0, 2)), (zeros(5, 3, 2 * piece, dtype=torch.uint8)[..., ::2],) * 2):
        with pytest.raises(ValueError):
            g.KvCacheFp4(K, V, 16, 64)
    with pytest.raises(g.GeloError):
        g.KvCacheFp4(good, good, 16, 48)


def test_adapters_are_described_by_their_tensors():
    A, B = zeros(7, 24, 64), zeros(7, 80, 8)
    s = g.Adapters(A, B, part_ends=[16, 48, 80]).struct
    assert (s.n_adapters, s.rank, s.n_parts, list(s.part_end)[:3]) == (7, 8, 3, [16, 48, 80])
    assert (s.a_stride, s.lda, s.b_stride, s.ldb, s.scale) == (24 * 64, 64, 640, 8, None)
    wide = zeros(7, 2, 40, 72)
    s = g.Adapters(wide[:, 0, :16, :64], zeros(7, 32, 24)[..., :16], scale=zeros(7, dtype=torch.float32)).struct
    assert (s.rank, s.n_parts, s.part_end[0], s.a_stride, s.lda, s.b_stride, s.ldb) == (16, 1, 32, 2 * 40 * 72, 72, 32 * 24, 24)
    s = g.Adapters(A.expand(7, 24, 64)[:1].expand(3, 24, 64), zeros(3, 80, 8), part_ends=(16, 48, 80)).struct
    assert s.a_stride == 0                                   # the same A for all


def test_adapters_that_are_refused():
    A, B = zeros(7, 24, 64), zeros(7, 80, 8)
    for bad in (dict(A=zeros(6, 24, 64)), dict(A=zeros(7, 16, 64)), dict(A=zeros(7, 24, 64, dtype=torch.float32)), dict(part_ends=[16, 48, 72]), dict(part_ends=[]),
                dict(A=zeros(7, 40, 64), part_ends=[16, 32, 48, 64, 80]), dict(A=torch.zeros((7, 24, 64), dtype=torch.bfloat16)),
                dict(A=zeros(7, 24, 128)[..., ::2]), dict(B=zeros(7, 8, 80).transpose(1, 2)), dict(scale=zeros(7)), dict(scale=zeros(6, dtype=torch.float32)),
                dict(scale=zeros(14, dtype=torch.float32)[::2]), dict(A=zeros(24, 64))):
        with pytest.raises(ValueError):
            g.Adapters(**{"A": A, "B": B, "part_ends": [16, 48, 80], **bad})
    with pytest.raises(TypeError):
        g.Adapters(zeros(7, 24, 64, dtype=torch.float16), zeros(7, 80, 8, dtype=torch.float16), part_ends=[16, 48, 80])


def test_calls_of_adapters_that_the_binding_refuses():
    """Before anything reaches the library (whose context is none here)."""
    ad = g.Adapters(zeros(7, 24, 64), zeros(7, 80, 8), part_ends=[16, 48, 80])
    H, Z, which = zeros(5, 64), zeros(5, 80), zeros(5, dtype=torch.int32)
    good = dict(H=H, which=which, Z=Z, base=None)
    for bad, kind in ((dict(H=zeros(5, 72)), g.GeloError), (dict(Z=zeros(4, 80)), g.GeloError), (dict(base=zeros(5, 88)), g.GeloError),
                      (dict(H=zeros(5, 64, dtype=torch.float32)), g.GeloError), (dict(base=zeros(5, 80, dtype=torch.float32)), g.GeloError),
                      (dict(which=zeros(4, dtype=torch.int32)), ValueError), (dict(which=zeros(5, dtype=torch.int64)), ValueError),
                      (dict(which=torch.zeros(5, dtype=torch.int32)), ValueError), (dict(H=torch.zeros((5, 64), dtype=torch.bfloat16)), ValueError),
                      (dict(Z=zeros(80, 5).t()), ValueError)):
        with pytest.raises(kind):
            g.gelo_adapt(None, adapters=ad, stream=0, **{**good, **bad})
    with pytest.raises(g.GeloError):                         # no context
        g.gelo_adapt(None, adapters=ad, stream=0, **good)


def test_calls_on_a_cache_of_4_bits_that_the_binding_refuses():
    piece = g.gelo_fp4_page_bytes(16, 64)
    pool = zeros(8, 2, piece, dtype=torch.uint8)
    cache = g.KvCacheFp4(pool, pool.clone(), 16, 64)
    batch = g.SeqBatch(zeros(3, dtype=torch.int32), zeros(3, 2, dtype=torch.int32), 32)
    Q, QKV = zeros(3, 256), zeros(3, 512)
    for call, kind in ((lambda: g.gelo_attention_fp4(None, Q, zeros(3, 256, dtype=torch.float32), 4, cache, batch, 1.0, stream=0), g.GeloError),
                       (lambda: g.gelo_attention_fp4(None, Q, zeros(3, 128), 4, cache, batch, 1.0, stream=0), g.GeloError),
                       (lambda: g.gelo_attention_fp4(None, Q, zeros(3, 256), 2, cache, batch, 1.0, stream=0), g.GeloError),
                       (lambda: g.gelo_attention_fp4(None, zeros(4, 256), zeros(4, 256), 4, cache, batch, 1.0, stream=0), g.GeloError),
                       (lambda: g.gelo_attention_fp4(None, Q, zeros(3, 256), 4, cache, g.SeqBatch(batch.kv_len, batch.page_table, 33), 1.0, stream=0), g.GeloError),
                       (lambda: g.gelo_rope_append_fp4(None, zeros(3, 520), 4, cache, batch, Q=Q, stream=0), g.GeloError),
                       (lambda: g.gelo_rope_append_fp4(None, QKV, 4, cache, batch, Q=zeros(3, 256, dtype=torch.float32), stream=0), ValueError),
                       (lambda: g.gelo_rope_append_fp4(None, QKV, 4, cache, batch, Q=Q, table=zeros(32, 32, 2), rot_dim=64, stream=0), ValueError),
                       (lambda: g.gelo_rope_append_fp4(None, torch.zeros((3, 512), dtype=torch.bfloat16), 4, cache, batch, Q=Q, stream=0), ValueError),
                       (lambda: g.gelo_cache_rows_fp4(None, cache, batch, stream=0), ValueError),
                       (lambda: g.gelo_cache_rows_fp4(None, cache, batch, zeros(3, 64), stream=0), ValueError),
                       (lambda: g.gelo_cache_rows_fp4(None, cache, batch, zeros(3, 128), zeros(3, 128, dtype=torch.float32), stream=0), ValueError),
                       (lambda: g.gelo_cache_rows_fp4(None, cache, batch, zeros(4, 128), stream=0), g.GeloError)):
        with pytest.raises(kind):
            call()


def test_every_call_wants_a_context():
    lib, P = g.load_library(), ctypes.c_void_p
    assert lib.gelo_rope_append_fp4(None, 1, 4, P(16), 512, None, None, 0, 0, None, 0, P(16), 256, None) == 1
    assert lib.gelo_cache_rows_fp4(None, 1, None, None, P(16), 128, None, 0, None) == 1
    assert lib.gelo_attention_fp4(None, 1, 4, P(16), 256, None, None, 1.0, 1, P(16), 256, None) == 1
    assert lib.gelo_adapt(None, 1, 4, 64, 64, P(16), 64, None, P(16), P(16), 64, P(16), 64, None) == 1
    assert lib.gelo_reserve_adapt(None, 4, 8, 1, 1) == 1


def test_reserved_workspace_of_adapters_serves_every_smaller_call():
    lib = ctypes.CDLL(g.LIB_PATH)
    needs, bound = lib["_ZN4gelo11adapt_needsEiiiiiii"], lib["_ZN4gelo21adapt_workspace_boundEiiii"]
    needs.restype = bound.restype = ctypes.c_size_t
    rng = random.Random(1)
    for _ in range(20000):
        n = int(2 ** rng.uniform(0, 15))
        rank, parts, count = 8 * rng.randint(1, 16), rng.randint(1, 4), int(2 ** rng.uniform(0, 15))
        reserved = bound(n, rank, parts, count)
        for _ in range(4):
            less = rng.choice([n, rng.randint(1, n), min(n, 256), min(n, 257)])
            d, p = 8 * rng.randint(1, 2000), 8 * rng.randint(2, 3000)
            got = needs(rng.randint(0, 1), less, d, p, rng.choice([8, rank]), rng.randint(1, parts), rng.choice([count, rng.randint(1, count)]))
            assert 0 < got <= reserved, (n, rank, parts, count, less, d, p)


def test_reserved_workspace_of_attention_serves_caches_of_4_bits():
    """gelo_reserve_attention sizes one workspace for both kinds of cache."""
    lib = ctypes.CDLL(g.LIB_PATH)
    needs, bound = lib["_ZN4gelo19attention_fp4_partsEiiiiiiiii"], lib["_ZN4gelo25attention_workspace_boundEi"]
    needs.restype = bound.restype = ctypes.c_size_t
    rng = random.Random(2)
    for _ in range(20000):
        d, hkv = rng.choice([64, 96, 128, 256]), rng.choice([1, 2, 3, 4, 8, 16, 32, 40])
        seqs, rows, kv = (int(2 ** rng.uniform(0, x)) for x in (9, 13, 20))
        got = needs(rng.randint(0, 1), rng.randint(0, 1), hkv * rng.choice([1, 2, 4, 7, 16]), hkv, d, seqs, seqs * rows if rng.random() < 0.7 else rows, rows, kv)
        assert got <= bound(d), (d, hkv, seqs, rows, kv)


def test_which_way_attention_over_4_bits_goes():
    """Few columns to a key head or many (1, 2: tiles in pairs), the cache cut (4), a head to a wave (8).  Measured, us, few and many: 1 x 100 rows of 32 heads of 128 6.2 and 10.3,
    16 x 32 rows on 512 keys, 12 heads of 64, 8.8 and 14.4, 8 x 128 on 512, 32 heads, 37.7 and 23.4, 8 x 512 118 and 45.7, 1 x 2000 32/8 113 and 62.8, 1 x 500 on 8500 8/8 of 64 39 and 35."""
    way = ctypes.CDLL(g.LIB_PATH)["_ZN4gelo17attention_fp4_wayEiiiiiiiii"]
    for want, args in ((0, (1, 1, 32, 32, 128, 1, 100, 100, 100)), (0, (1, 1, 12, 12, 64, 16, 512, 32, 512)), (1, (1, 1, 32, 32, 128, 8, 1024, 128, 512)), (2, (1, 1, 32, 32, 128, 8, 4096, 512, 512)),
                       (4, (1, 1, 32, 8, 128, 3, 3, 1, 32768)), (8, (1, 1, 32, 32, 128, 64, 64, 1, 4096)), (0, (0, 1, 32, 32, 128, 64, 64, 1, 4096)), (8, (0, 1, 32, 32, 64, 64, 64, 1, 4096)),
                       (0, (0, 1, 32, 32, 128, 8, 4096, 512, 512)), (5, (1, 1, 8, 8, 64, 1, 500, 500, 8500))):
        assert way(*args) == want, args


def test_which_way_adapters_go():
    """Rows by themselves, groups as they come (1), groups put in order (2).  Measured, us: see kRowsRead and few_adapters in adapt.hip."""
    way = ctypes.CDLL(g.LIB_PATH)["_ZN4gelo9adapt_wayEiiiiiii"]
    for want, args in ((0, (1, 64, 4096, 12288, 16, 3, 48)), (0, (1, 96, 4096, 12288, 16, 3, 1)), (1, (1, 128, 4096, 12288, 16, 3, 1)), (0, (1, 128, 4096, 12288, 16, 3, 64)),
                       (2, (1, 192, 4096, 12288, 16, 3, 64)), (1, (1, 64, 4096, 4096, 128, 1, 1)), (0, (1, 1024, 1024, 1024, 8, 1, 4)), (2, (1, 1024, 4096, 12288, 16, 3, 8)),
                       (1, (1, 4096, 4096, 12288, 16, 3, 8)), (2, (1, 4096, 2048, 2048, 64, 1, 8)), (1, (1, 4096, 2048, 2048, 64, 1, 4)), (2, (1, 4096, 4096, 12288, 16, 3, 9)), (0, (1, 4096, 4096, 12288, 16, 3, 12288))):
        assert way(*args) == want, args
