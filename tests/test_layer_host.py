"""The host's side of the operators between two projections: what the binding makes of tensors, and what the library reckons from
sizes.  Nothing here launches a kernel or needs a GPU."""
import ctypes
import os
import random
import subprocess
import sys

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


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_rows_of_a_page_table_lie_where_its_strides_say():
    """An expanded table (all sequences share a row) has stride 0, and overlapping rows less than their width: a row width in their place would
    have the kernels read behind the tensor."""
    def ld(table, n_seqs):
        return g.SeqBatch(on_gpu(ints(n_seqs)), on_gpu(table), 32).struct.table_ld
    assert ld(ints(1, 6).expand(4, 6), 4) == 0                     # which the library refuses
    assert ld(ints(64).as_strided((4, 6), (2, 1)), 4) == 2
    assert ld(ints(4, 6), 4) == 6 and ld(ints(4, 9)[:, :6], 4) == 9 and ld(ints(4, 1), 4) == 1
    assert ld(ints(1, 6).as_strided((1, 6), (0, 1)), 1) == 6       # the stride of one row says nothing


@pytest.mark.parametrize("wrong", ["on the host", "strided"])
def test_a_prepared_weight_that_the_kernels_cannot_read_is_refused(wrong):
    """Before anything reaches the library (whose context is none here: it would refuse in its own way)."""
    n, d, p = 4, 128, 8
    size = g.gelo_fp8_weight_bytes(d, p)
    Wq = torch.zeros(size, dtype=torch.uint8) if wrong == "on the host" else on_gpu(torch.zeros(2 * size, dtype=torch.uint8)[::2])
    codes, scales = on_gpu(torch.zeros((n, d), dtype=torch.uint8)), on_gpu(torch.zeros(n))
    U, Y = (on_gpu(torch.zeros((n, w), dtype=torch.bfloat16)) for w in (d, p))
    with pytest.raises(ValueError):
        g.gelo_project_fp8_codes(None, codes, scales, Wq, p, Y, stream=0)
    with pytest.raises(ValueError):
        g.gelo_project_fp8(None, U, Wq, p, Y, stream=0)


def reckoned(hook, *args):
    """What a hook of the library returns, asked in a process of its own (a division by zero ends one)."""
    code = f"import ctypes; print(ctypes.CDLL({g.LIB_PATH!r})[{hook!r}](*{args!r}))"
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (hook, args, r.returncode)
    return int(r.stdout)


WAY, FLOAT_WAY = "_ZN4gelo13attention_wayEiiiiiiiii", "_ZN4gelo19attention_float_wayEiiiiiiii"


@pytest.mark.parametrize("heads,max_rows", [(64, 2 ** 30), (64, 2 ** 30 + 16), (64, 2 ** 30 - 1), (32, 2147418111), (1, 2147418111)])
def test_a_bound_of_rows_far_above_them_plans_as_the_rows_do(heads, max_rows):
    """Rows times heads to a key head pass 32 bits there."""
    for rows in (16, 100, 4096):
        for causal in (0, 1):
            for bf16 in (0, 1):
                assert reckoned(WAY, bf16, causal, heads, 1, 128, 1, rows, max_rows, 4096) == reckoned(WAY, bf16, causal, heads, 1, 128, 1, rows, rows, 4096) >= 0
            assert reckoned(FLOAT_WAY, causal, heads, 1, 128, 1, rows, max_rows, 4096) == reckoned(FLOAT_WAY, causal, heads, 1, 128, 1, rows, rows, 4096) >= 0
    assert reckoned(WAY, 1, 1, heads, 1, 128, 1, 2 ** 23 + 1, max_rows, 4096) == -1         # rows' heads beyond one launch
    with pytest.raises(ValueError):
        g.SeqBatch(on_gpu(ints(1)), on_gpu(ints(1, 6)), 32, row_start=on_gpu(ints(2)), max_rows=2 ** 32 + 1)


def test_a_norm_of_the_most_rows_is_a_launch_of_at_most_2_to_the_31_threads():
    """Threads to a row as the launches of norm.hip have them, for d up to the second number of each pair."""
    most = ctypes.CDLL(g.LIB_PATH)["_ZN4gelo18rms_norm_most_rowsEi"]
    first = 8
    for threads, last in ((64, 512), (256, 2048), (512, 4096), (256, 8192), (1024, 65536)):
        for d in (first, last):
            assert 2 ** 20 < most(d) and most(d) * threads <= 2 ** 31, d
        first = last + 8


def test_the_workspace_that_is_reserved_is_enough_for_any_batch():
    """gelo_reserve_attention promises that no call allocates after it: rows of one sequence or many, cut caches, and more rows than the sequences
    may bring (a batch padded for a captured launch)."""
    lib = ctypes.CDLL(g.LIB_PATH)
    need, most = lib["_ZN4gelo15attention_partsEiiiiiiiii"], lib["_ZN4gelo25attention_workspace_boundEi"]
    need.restype = most.restype = ctypes.c_size_t
    assert need(1, 1, 32, 8, 128, 1, 4096, 1, 32768) == need(1, 1, 32, 8, 128, 1, 1, 1, 32768) > 0
    rng, cut = random.Random(1), 0
    for _ in range(20000):
        hkv, d = rng.choice([1, 2, 5, 8, 32]), rng.choice([64, 96, 128, 256])
        hq, seqs, rows = hkv * rng.choice([1, 2, 4, 7, 16]), int(2 ** rng.uniform(0, 8)), int(2 ** rng.uniform(0, 13))
        n_rows = min(rng.choice([seqs, seqs * rows, max(rows, seqs), int(2 ** rng.uniform(0, 15))]), 2 ** 23 // hq)
        size = need(rng.randint(0, 1), rng.randint(0, 1), hq, hkv, d, seqs, n_rows, rows, int(2 ** rng.uniform(4, 20)))
        assert size <= most(d), (hq, hkv, d, seqs, n_rows, rows)
        cut += size > 0
    assert cut > 1000


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_a_torch_without_its_private_names(missing):
    """The binding imports, and the current stream comes from torch's public call."""
    code = f"""
import torch
if hasattr(torch._C, {missing!r}):
    delattr(torch._C, {missing!r})
from paper_2603_05035_amd import binding
class Stream:
    cuda_stream = 77
torch.cuda.current_stream = Stream
assert binding._stream(None).value == 77 and binding._stream(Stream()).value == 77 and binding._stream(5).value == 5
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stderr[-2000:]


def test_calls_of_other_rows_do_not_change_a_description_in_use(monkeypatch):
    """Threads that share a batch: a call of 7 rows comes in while one of 5 rows is in the library."""
    K, V = (on_gpu(torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16)) for _ in range(2))
    batch = g.SeqBatch(on_gpu(ints(1)), on_gpu(ints(1, 2)), 32, row_start=on_gpu(ints(2)), max_rows=7)
    cache, seen = g.KvCache(K, V), []

    def attention(rows):
        Q, O = (on_gpu(torch.zeros((rows, 64), dtype=torch.bfloat16)) for _ in range(2))
        g.gelo_attention(None, Q, O, 1, cache, batch, 1.0, stream=0)

    class Library:
        @staticmethod
        def gelo_attention(*args):
            described = g._SeqBatchStruct.from_address(args[6])
            seen.append(described.n_rows)
            if len(seen) == 1:
                attention(7)
            seen.append(described.n_rows)
            return g.GELO_OK

    monkeypatch.setattr(g, "load_library", Library)
    attention(5)
    assert seen == [5, 7, 7, 5]


def test_which_way_float_attention_goes():
    """attention_way tells the kernels of bfloat16 apart (float is 0 or cut there, whichever kernel takes it); which one takes float is
    attention_float_way's to say: 1 by tiles of 64 columns, 0 by 16, plus 4 where the cache is cut.  Measured, us, 16 columns and 64: 8 x 512 rows of 32 heads
    of 128 478 and 291, 2 x 512 on 2000 of 8 heads 99 and 93, 1 x 2000 of 8 heads 148 and 162."""
    for want, args in ((1, (1, 32, 32, 128, 8, 4096, 512, 512)), (5, (1, 8, 8, 128, 2, 1024, 512, 2000)), (0, (1, 8, 8, 128, 1, 2000, 2000, 2000)),
                       (0, (1, 32, 32, 64, 8, 4096, 512, 512)), (0, (1, 32, 32, 256, 8, 4096, 512, 512)), (4, (1, 32, 8, 128, 3, 3, 1, 32768)),
                       (0, (1, 32, 32, 128, 64, 64, 1, 4096))):
        assert reckoned(FLOAT_WAY, *args) == want, args
        assert reckoned(WAY, 0, *args) == want & 4, args


@pytest.mark.parametrize("max_kv_len", [2 ** 30 + 1, 2 ** 31 - 65537])
@pytest.mark.parametrize("n_seqs,heads", [(64, 32), (1, 1), (1, 8), (3, 50)])
def test_a_bound_of_lengths_near_2_to_the_31_is_cut_as_others_are(max_kv_len, n_seqs, heads):
    """A bound and the chunk together pass 32 bits.  The parts that a call needs are those of its chunks: none for a whole cache, and no fewer with a longer bound."""
    def parts(most):
        return reckoned("_ZN4gelo15attention_partsEiiiiiiiii", 1, 1, heads, heads, 64, n_seqs, n_seqs, 1, most)
    few = parts(2 ** 29)
    assert parts(max_kv_len) == few and (few > 0) == (n_seqs * heads <= 256)
    assert reckoned(WAY, 1, 1, heads, heads, 64, n_seqs, n_seqs, 1, max_kv_len) == (4 if few else 0)
