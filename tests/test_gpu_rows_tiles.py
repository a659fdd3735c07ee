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


# ---- the sum of a token's slots -------------------------------------------------

@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 8])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_combine_longest_rows(n, dtype):
    """Rows of the most elements that a call takes: the last 16 bytes of each are whole or
    not, and what lies behind them is neither read into the sum nor written."""
    Z = torch.ones(2 * n, dtype=dtype, device="cuda").view(2, n)
    Z[0, -9:] = torch.arange(2, 11, device="cuda")
    whole = torch.full((n + 64,), 7.0, dtype=dtype, device="cuda")
    out = whole[:n].view(1, n)
    ig.combine(Z, torch.tensor([[1.0, 2.0]], device="cuda"), out=out)
    assert bool((whole[n:] == 7).all())
    assert out[0, -9:].tolist() == [float(x + 2) for x in range(2, 11)]
    assert bool((out[0, :1 << 30] == 3).all()) and bool((out[0, 1 << 30:-9] == 3).all())


@pytest.mark.parametrize("top_k", [1, 7, 8, 9, 16, 65])
@pytest.mark.parametrize("tokens, n", [(1100, 2048), (300, 8192)])
def test_combine_many_values(tokens, n, top_k):
    """Workgroups of 256 threads, with slots to the left and right of the eights."""
    g = torch.Generator(device="cuda").manual_seed(top_k)
    Z = torch.randn(tokens * top_k, n, generator=g, device="cuda").bfloat16()
    w = torch.randn(tokens, top_k, generator=g, device="cuda")
    ids = torch.where(torch.rand(tokens, top_k, generator=g, device="cuda") < 0.2, -1, 3).int()
    z = Z.double().view(tokens, top_k, n) * torch.where(ids < 0, 0.0, w.double())[:, :, None]
    want, size = z.sum(1), z.abs().sum(1)
    got = ig.combine(Z, w, ids=ids)
    bound = (top_k + 2) * STEP[F32] * size + STEP[BF16] * want.abs() * 1.001 + 2.0 ** -134
    assert bool(((got.double() - want).abs() <= bound).all())


# ---- route -------------------------------------------------------------------

@pytest.mark.parametrize("default", [torch.bfloat16, torch.float16, torch.float64])
def test_route_under_another_default_type(default):
    x = torch.randn(40, 70, device="cuda")
    want = ig.route(x, 5)
    try:
        torch.set_default_dtype(default)
        got = ig.route(x, 5, stream=torch.cuda.current_stream())
    finally:
        torch.set_default_dtype(F32)
    assert all(torch.equal(g, w) and g.dtype == w.dtype for g, w in zip(got, want))
