"""The operators of include/igemm_rows.h on the GPU: sizes that run the large tiles
and the forms that the sizes of test_gpu_rows.py do not reach, against the same
references (rows_reference.py) with the same tolerances."""
import numpy as np
import pytest
import torch

import paper_2302_07594_amd as ig
import rows_reference as ref
from test_gpu_rows import BF16, F16, F32, INF, STEP, check_grouped, close, cuda, ints, rounded, split

pytestmark = pytest.mark.gpu


def test_offsets_that_do_not_ascend_over_many_columns():
    """Row tiles times column tiles of these offsets pass 2^31, with an order: nothing
    beside out is written, and the values there are one product's."""
    rows, groups, n = 262144, 8192, 16640 + 40
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda").repeat(groups // 2)
    off = torch.cat([off, off[:1]])
    order = torch.arange(rows, dtype=torch.int32, device="cuda") % 64
    a = torch.ones(1, 1, dtype=torch.int8, device="cuda")
    b = torch.ones(1, 1, n, dtype=torch.int8, device="cuda").expand(groups, 1, n)
    whole = torch.full((64 + 16, n), 7.0, dtype=BF16, device="cuda")
    out = whole[8:-8]
    ig.grouped_i8(a, b, off, order, slots=rows, scatter=True, out=out)
    torch.cuda.synchronize()
    assert bool((whole[:8] == 7).all()) and bool((whole[-8:] == 7).all())
    assert bool(((out == 1) | (out == 7)).all())
