"""Books of the paged cache whose lengths are not lengths."""
import pytest
import torch

import paper_2607_22634_amd as P
from test_gpu_paged import flag, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("length", [-1, 65, 1 << 30, -(1 << 31), 2 ** 31 - 1])
def test_trim_leaves_sequences_of_impossible_lengths_alone(length):
    """Four columns of 16 positions hold 64."""
    table0 = [[0, 1, 2, 3], [4, 5, 6, 7], [8, 9, 10, -1]]
    refs, table, ctx, f = ints([1] * 12), ints(table0), ints([64, length, 40]), flag()
    P.presto_pages_trim(refs, table, ctx, 16, 20, 0, flags=f)
    assert f.item() == P.PRESTO_FLAG_BAD_SEQ
    assert table.tolist() == [[-1, -1, 2, 3], table0[1], [-1, 9, 10, -1]]
    assert refs.tolist() == [0, 0, 1, 1, 1, 1, 1, 1, 0, 1, 1, 1]
    assert ctx.tolist() == [64, length, 40]
    f = flag()
    P.presto_pages_trim(refs, table, ints([0, 64, 0]), 16, 20, 0, flags=f)
    torch.cuda.synchronize()
    assert f.item() == 0 and table.tolist()[1] == [-1, -1, 6, 7]
