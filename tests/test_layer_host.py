"""The host's side of the operators between two projections: what the binding makes of tensors, and what the library reckons from
sizes.  Nothing here launches a kernel or needs a GPU."""
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
