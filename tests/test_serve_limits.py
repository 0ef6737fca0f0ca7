"""Adapters and the cache of 4 bits at the ends of what a call may say: what the library reckons on the host.  Nothing here launches a kernel or needs a GPU."""
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import serve_oracle as so
from paper_2603_05035_amd import binding as g

ROWS = """
import ctypes, sys
lib = ctypes.CDLL(sys.argv[1])
way, needs, fits = lib["_ZN4gelo9adapt_wayEiiiiiii"], lib["_ZN4gelo11adapt_needsEiiiiiii"], lib["_ZN4gelo10adapt_fitsERKNS_5AdaptEi"]
needs.restype, fits.restype = ctypes.c_size_t, ctypes.c_bool
P, I, L = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
class Adapt(ctypes.Structure):
    _fields_ = [("H", P), ("ldh", L), ("base", P), ("ldb", L), ("Z", P), ("ldz", L), ("A", P), ("a_stride", L), ("lda", L), ("B", P), ("b_stride", L), ("ldbw", L),
                ("scale", P), ("which", P), ("n", I), ("d", I), ("p", I), ("rank", I), ("n_parts", I), ("n_adapters", I), ("part_end", I * 4), ("workspace", P)]
adapters, d, p = (int(x) for x in sys.argv[2:])
for n in (2 ** 31 - 1, 2 ** 31 - 15, 2 ** 31 - 31, 2 ** 31 - 32, 2 ** 31 - 62, 2 ** 31 - 63, 2 ** 31 - 64, 2 ** 30, 2 ** 28 + 1):
    for bf16 in (0, 1):
        o = Adapt(n=n, d=d, p=p, rank=16, n_parts=1, n_adapters=adapters)
        assert not fits(ctypes.byref(o), bf16), n            # refused
        assert way(bf16, n, d, p, 16, 1, adapters) in (0, 1, 2)
        assert needs(bf16, n, d, p, 16, 1, adapters) >= n * 16 * 4
assert fits(ctypes.byref(Adapt(n=4096, d=d, p=p, rank=16, n_parts=1, n_adapters=adapters)), 1)
"""


@pytest.mark.parametrize("adapters", [1, 20, 12287, 12288, 2 ** 31 - 1])
@pytest.mark.parametrize("d,p", [(4096, 4096), (8, 8)])
def test_numbers_of_rows_at_the_end_of_32_bits(adapters, d, p):
    """No launch has so many rows: they are refused, by sums that stay what they are.  (In a process of its own: a division by zero would end it.)"""
    r = subprocess.run([sys.executable, "-c", ROWS, g.LIB_PATH, str(adapters), str(d), str(p)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stdout[-2000:])


class OnGpu(torch.Tensor):
    """A host tensor that says it lives on the GPU: for code that looks at shapes and strides only."""

    @property
    def is_cuda(self):
        return True


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


@pytest.mark.parametrize("call", ["append", "rows", "attention"])
def test_a_cache_of_values_is_not_one_of_4_bits(call, monkeypatch):
    """Nothing reaches the library: with the address of the other kind's structure it would write codes over values."""
    def load():
        raise AssertionError("reached the library")
    piece = g.gelo_fp4_page_bytes(16, 64)
    pool, bytes_ = zeros(8, 2, 16, 64), zeros(8, 2, piece, dtype=torch.uint8)
    values, codes = g.KvCache(pool, pool.clone()), g.KvCacheFp4(bytes_, bytes_.clone(), 16, 64)
    batch = g.SeqBatch(zeros(3, dtype=torch.int32), zeros(3, 2, dtype=torch.int32), 32)
    Q, QKV, K = zeros(3, 256), zeros(3, 512), zeros(3, 128)
    run = {"append": lambda cache: g.gelo_rope_append_fp4(None, QKV, 4, cache, batch, Q=Q, stream=0),
           "rows": lambda cache: g.gelo_cache_rows_fp4(None, cache, batch, K, stream=0),
           "attention": lambda cache: g.gelo_attention_fp4(None, Q, zeros(3, 256), 4, cache, batch, 1.0, stream=0)}[call]
    monkeypatch.setattr(g, "load_library", load)
    for cache in (values, None, bytes_):
        with pytest.raises(TypeError):
            run(cache)
    with pytest.raises(AssertionError):                      # the right kind does
        run(codes)


@pytest.mark.parametrize("seed", range(4))
def test_how_far_a_value_of_4_bits_is_off(seed):
    """As include/gelo.h says it, at the ends of the scales too (the kernels' codes are compared with the oracle's to the bit where there is a GPU)."""
    rng = np.random.default_rng(seed)
    most, least = 7 * 2.0 ** 125, 3.5 * 2.0 ** -110
    tops = np.concatenate((most * np.array([1 - 2.0 ** -20, 1.0, 1 + 2.0 ** -20, 8 / 7, 1.6]), least * np.array([2.0, 1 + 2.0 ** -20, 1.0, 0.6, 0.1, 0.05, 1e-4]),
                           10.0 ** rng.uniform(-32, 38, 40)))
    x = rng.uniform(-1, 1, (len(tops), 32))
    x[:, 7] = 1
    x = x / np.abs(x).max(1, keepdims=True) * tops[:, None]
    codes, scales = so.hold(x)
    off, step = np.abs(so.held(codes, scales) - x), 2.0 ** (scales[:, 0] - 127.0)
    inside = np.abs(x) <= most
    assert (off <= step[:, None])[inside].all() and (np.abs(so.held(codes, scales))[~inside] == 6 * 2.0 ** 125).all() and not inside.all()
    usual = (tops > least) & (tops <= most)
    assert (step[usual] >= tops[usual] / 7 * (1 - 2.0 ** -50)).all() and (step[usual] < tops[usual] * 2 / 7).all()
    small = tops <= least
    assert small.sum() == 5 and (step[small] == 2.0 ** -110).all() and (off[small] <= 2.0 ** -111).all()
    assert (so.held(codes, scales)[np.abs(x) <= 2.0 ** -112] == 0).all()
    # (at the ends a value can be off by more than the step, and the step be more than two sevenths)
    assert (off[3:5] > step[3:5, None]).any(1).all() and (step[8:12] > tops[8:12] * 2 / 7).all()
