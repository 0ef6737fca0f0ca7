"""The host's side of the operators between two projections: what the binding makes of tensors, and what the library reckons from
sizes.  Nothing here launches a kernel or needs a GPU."""
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
