"""The operators of include/igemm_rows.h on the GPU: sizes that run the large tiles and the
forms that the sizes of test_gpu_rows.py do not reach, against definitions in float64,
with that file's tolerances."""
import numpy as np
import pytest
import torch

import paper_2302_07594_amd as ig
from rows_tiles import ADAPTERS, GROUPED
from test_gpu_rows import (BF16, F16, F32, INF, STEP, check_adapters, check_route, cuda, ints,
                           make_adapters, strided)

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


@pytest.mark.parametrize("bias", [False, True])
def test_route_smallest_sigmoids(bias):
    """Logits whose sigmoid lies at the end of 64-bit floating point: in the order of their
    scores, with the weights of a normalised choice."""
    g = torch.Generator().manual_seed(5)
    x = -(709.7 - 0.6 * torch.rand(40, 64, generator=g))
    x[20:] = -(300.0 + 400.0 * torch.rand(20, 64, generator=g))
    x[38] = -(705.0 + 10.0 * torch.rand(64, generator=g))
    x[39] = -41.0 + 2.0 * torch.rand(64, generator=g)
    b = torch.zeros(64) if bias else None
    check_route(x.cuda(), 6, bias=b, groups=4, top_groups=2, group_best=2, score="sigmoid")
    if bias:
        check_route(x.cuda(), 6, bias=b, score="sigmoid")


# ---- adapters ------------------------------------------------------------------

def same_infinities(got, want, bound, what):
    """Infinities and NaN where the formula has them, and the rest within bound."""
    g = got.double()
    for name, f in (("NaN", torch.isnan), ("infinity", torch.isposinf),
                    ("-infinity", torch.isneginf)):
        bad = f(g) != f(want)
        assert not bool(bad.any()), (what, name, int(bad.sum()), bad.nonzero()[:4].tolist(),
                                     g[bad][:4].tolist(), want[bad][:4].tolist())
    ok = want.isfinite()
    assert bool(((g - want).abs() <= bound)[ok].all()), what


# u's lower parts, or a float16 weight's second one, are 0 for values of few bits: the sizes
# run the row kernels and their k slices, tiles of 32, 128 and 256 rows, through
# registers (odd rows) and by DMA.
@pytest.mark.parametrize("m, n, k, rank", [
    (3, 40, 64, 5), (3, 64, 2048, 16), (130, 72, 64, 33), (131, 90, 33, 40), (2048, 2048, 64, 24),
    (2050, 2047, 65, 24), (4096, 4096, 64, 16)])
@pytest.mark.parametrize("wt", [BF16, F16])
def test_adapters_with_infinite_factors(m, n, k, rank, wt):
    """An infinite weight or an infinite u gives what the formula gives, whichever kernel
    runs: infinities of the product's sign, NaN for 0 times infinity and for
    infinities of both signs."""
    rng = np.random.default_rng(m + n)
    A = np.zeros((m, k), np.int8)
    A[:, :4] = rng.choice([-2, -1, 1, 4, 0, 3, 119], (m, 4), p=[.2, .2, .2, .2, .05, .1, .05])
    B = ints(rng, k, n, lo=-3, hi=3)
    down = np.zeros((3, rank, k))
    down[:, np.arange(rank), np.arange(rank) % 4] = rng.choice([0.5, 1.0, -2.0, 1.7], (3, rank))
    up = rng.choice([0.0, 1.0, -0.5, 0.7], (3, n, rank))
    up[0, :, 0] = rng.choice([1.0, np.inf, -np.inf, 0.3], n)
    up[1, : n // 2, rank - 1] = np.inf
    down, up = torch.from_numpy(down).to(wt), torch.from_numpy(up).to(wt)
    scaling = np.array([1.0, 0.75, np.inf], np.float32)
    ids = (np.arange(m) % 4 - 1).astype(np.int32)
    got = ig.adapters_i8(cuda(A), cuda(B), cuda(ids), down.cuda(), up.cuda(),
                         scaling=cuda(scaling), out_dtype=F32)
    a = torch.from_numpy(A).double()
    base = (a @ torch.from_numpy(B).double()).cuda()
    want, reach = base.clone(), torch.zeros_like(base)
    for w in range(3):
        rows = torch.from_numpy(np.flatnonzero(ids == w)).cuda()
        u = (a[rows.cpu()] @ down[w].double().T * float(scaling[w])).cuda()
        v = up[w].double().cuda()
        for r in range(rank):     # (a product of infinities by its definition, term by term)
            term = u[:, r:r + 1] * v[None, :, r]
            want[rows] += term
            reach[rows] += term.abs()
    bound = want.abs() * 8 * STEP[F32] + 4 * STEP[F32] * base.abs() + \
        (k + rank + 8) * STEP[F32] * reach + 2.0 ** -22 * reach
    same_infinities(got, want, bound, (m, n, k, rank, wt))


@pytest.mark.parametrize("m", [3, 130, 4096])
@pytest.mark.parametrize("wt", [BF16, F16])
def test_adapters_with_small_u(m, wt):
    """u down to the smallest floats, of one bit and of 24: within 2^-134, and infinite
    against an infinite weight down to 2^-100."""
    n = 4096 if m == 4096 else 64
    a = torch.ones(m, 4, dtype=torch.int8, device="cuda")
    b = torch.zeros(4, n, dtype=torch.int8, device="cuda")
    ids = torch.zeros(m, dtype=torch.int32, device="cuda")
    down = torch.zeros(1, 16, 4, dtype=wt, device="cuda")
    down[:, 0, 0] = 1
    up = torch.zeros(1, n, 16, dtype=wt, device="cuda")
    up[:, : n // 2, 0], up[:, n // 2:, 0] = 1, INF
    for e in (0, -50, -100, -101, -110, -126, -133, -149):
        for mantissa in (1.0, 1.0 + 2.0 ** -23, 2.0 - 2.0 ** -23, 1.5):
            u = np.float32(mantissa * 2.0 ** e)
            got = ig.adapters_i8(a, b, ids, down, up, out_dtype=F32,
                                 scaling=torch.tensor([u], dtype=F32, device="cuda"))
            left, right = got[:, : n // 2], got[:, n // 2:]
            assert bool(((left.double() - float(u)).abs() <= 2.0 ** -134).all()), (e, mantissa)
            assert e < -100 or bool((right == INF).all()), (e, mantissa)


# ---- autograd ------------------------------------------------------------------

def layer_calls():
    """(name of an operand, the call with it, the operand) of each call, plain and with a
    stream (the binding's way and the Python code's)."""
    d = dict(device="cuda")
    a = torch.ones(6, 32, dtype=torch.int8, **d)
    b = torch.ones(2, 32, 16, dtype=torch.int8, **d)
    off = torch.tensor([0, 2, 6], dtype=torch.int32, **d)
    ids = torch.zeros(6, dtype=torch.int32, **d)
    sa, w = torch.rand(6, **d), torch.rand(3, 2, **d)
    z, y = torch.rand(6, 16, **d), torch.rand(3, 16, **d)
    down, up = torch.rand(1, 8, 32, **d).bfloat16(), torch.rand(1, 16, 8, **d).bfloat16()
    scaling = torch.rand(1, **d)
    out = torch.zeros(6, 16, **d)
    for kw in ({}, {"stream": torch.cuda.current_stream()}):
        yield "logits", lambda t, kw=kw: ig.route(t, 2, **kw)[1], torch.rand(5, 9, **d)
        yield "bias", lambda t, kw=kw: ig.route(torch.rand(5, 9, **d), 2, bias=t, **kw)[0], \
            torch.rand(9, **d)
        yield "scale_a", lambda t, kw=kw: ig.grouped_i8(a, b, off, scale_a=t, out=out, **kw), sa
        yield "out", lambda t, kw=kw: ig.grouped_i8(a, b, off, out=t, **kw), z
        yield "Z", lambda t, kw=kw: ig.combine(t, w, out=y, **kw), z
        yield "weights", lambda t, kw=kw: ig.combine(z, t, out=y, **kw), w
        yield "base", lambda t, kw=kw: ig.combine(z, w, base=t, out=t.detach().clone(), **kw), y
        yield "out", lambda t, kw=kw: ig.combine(z, w, out=t, **kw), y.clone()
        for name, t in (("down", down), ("up", up), ("scaling", scaling)):
            yield name, lambda t, kw=kw, name=name: ig.adapters_i8(
                a, b[0], out=out, **dict(dict(ids=ids, down=down, up=up, scaling=scaling),
                                         **{name: t}), **kw), t
        yield "out", lambda t, kw=kw: ig.adapters_i8(a, b[0], ids, down, up, out=t, **kw), z.clone()


def test_no_tangent_is_dropped_in_silence():
    fw = torch.autograd.forward_ad
    for name, call, t in layer_calls():
        with fw.dual_level():
            dual = fw.make_dual(t, torch.ones_like(t))
            with pytest.raises(ValueError, match=f"detach {name}"):
                call(dual)
            with torch.no_grad(), pytest.raises(ValueError, match=f"detach {name}"):
                call(dual)
            call(dual.detach())
            call(t)
        call(t)


def test_outputs_that_autograd_saved():
    """A backward pass over a value that a call has overwritten is refused by torch."""
    for name, call, t in layer_calls():
        if name != "out":
            continue
        version = t._version
        x = torch.rand_like(t).requires_grad_()
        y = (x * t).sum()                  # t is saved for x's gradient
        with torch.no_grad():
            call(t)
        assert t._version == version + 1
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
        with torch.inference_mode():
            call(torch.empty_like(t))


# ---- every tile, with values that tell rows, columns and groups apart ---------------

def gpu_ints(g, *shape):
    return torch.empty(shape, dtype=torch.int8, device="cuda").random_(-128, 128, generator=g)


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def uneven(rng, rows, groups):
    """Offsets of groups of very different rows, one of them with half of all (more than
    eight row tiles of the large sizes) and some with none."""
    share = rng.random(groups) ** 3 * (rng.random(groups) < 0.8)
    share[rng.integers(groups)] = share.sum() + 0.1
    cuts = np.floor(np.cumsum(share / share.sum())[:-1] * rows).astype(np.int64)
    return np.concatenate([[0], cuts, [rows]]).astype(np.int32)


def exact_grouped(a, b, offsets, order, sa, sb, slots, scatter, out):
    """out (float64) where positions lead, by exact products in float64."""
    for g in range(b.shape[0]):
        i = torch.arange(int(offsets[g]), int(offsets[g + 1]), device="cuda")
        if len(i) == 0:
            continue
        s = i if order is None else order[i].long()
        ra = i if slots == 0 else s // slots
        y = a[ra].double() @ b[g].double()
        y = y * sa.double()[ra, None] * sb.double()[g]
        out[s if scatter else i] = y
    return out


def within(got, want, bound, what=""):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), bad.nonzero()[:4].tolist(),
                                 got[bad][:4].tolist(), want[bad][:4].tolist())


@pytest.mark.parametrize("way", ["plain", "gather", "scatter"])
@pytest.mark.parametrize("rows, n, k, groups", GROUPED)
def test_grouped_tiles(rows, n, k, groups, way):
    rng, g = np.random.default_rng(rows + n + k), generator(rows * 7 + n)
    dtype = {"plain": F32, "gather": BF16, "scatter": F16}[way]
    offsets = uneven(rng, rows, groups)
    slots = 2 if way == "gather" else 0
    a_rows = (rows + 1) // 2 if slots else rows
    a, b = gpu_ints(g, a_rows, k), gpu_ints(g, groups, k, n)
    sa = torch.rand(a_rows, generator=g, device="cuda") * 1e-3 + 1e-4
    sb = torch.rand(groups, n, generator=g, device="cuda") * 1e-2 + 1e-3
    order = None if way == "plain" else \
        torch.randperm(rows, generator=g, device="cuda").int()
    out = torch.full((rows + 2, n), 7.0, dtype=dtype, device="cuda")
    got = ig.grouped_i8(a, b, cuda(offsets), order, sa, sb, slots=slots,
                        scatter=way == "scatter", out=out)
    assert got is out
    want = exact_grouped(a, b, offsets, order, sa, sb, slots, way == "scatter",
                         torch.full(out.shape, 7.0, dtype=torch.float64, device="cuda"))
    tiny = {F32: 2.0 ** -150, BF16: 2.0 ** -134, F16: 2.0 ** -25}[dtype]
    within(out, want, want.abs() * (3 * STEP[F32] + STEP[dtype]) * 1.001 + tiny)
    assert bool((out[rows:] == 7).all())


@pytest.mark.parametrize("rows, n, k, groups", [s for s in GROUPED if s[0] >= 900])
def test_projection_tiles(rows, n, k, groups):
    """The projection alone at the same sizes."""
    g = generator(rows + n)
    a, b = gpu_ints(g, rows, k), gpu_ints(g, k, n)
    sa = torch.rand(rows, generator=g, device="cuda") + 0.1
    sb = torch.rand(n, generator=g, device="cuda") + 0.1
    want = (a.double() @ b.double()) * sa.double()[:, None] * sb.double()
    got = ig.adapters_i8(a, b, scale_a=sa, scale_b=sb, out_dtype=F32)
    within(got, want, want.abs() * 4 * STEP[F32] * 1.001)


def adapter_terms(a, b, ids, down, up, sa, sb, ranks, scaling):
    """As rows_reference.adapters: (out, base, reach, spread), in float64 on the GPU."""
    a64 = a.double()
    base = (a64 @ b.double()) * sa.double()[:, None] * sb.double()
    out, reach, spread = base.clone(), torch.zeros_like(base), torch.zeros_like(base)
    for w in range(down.shape[0]):
        i = (ids == w).nonzero().flatten()
        r = min(max(int(ranks[w]), 0), down.shape[1])
        if len(i) == 0 or r == 0:
            continue
        f = (float(scaling[w]) * sa[i].double())[:, None]
        d, v = down[w, :r].double(), up[w, :, :r].double()
        u = a64[i] @ d.T.contiguous() * f
        out[i] += u @ v.T.contiguous()
        reach[i] = ((a64[i].abs() @ d.abs().T.contiguous()) * f.abs()) @ v.abs().T.contiguous()
        spread[i] = u.abs().amax(1, keepdim=True) * v.abs().sum(1)
    return out, base, reach, spread


@pytest.mark.parametrize("wt, dtype", [(BF16, F32), (F16, F32), (BF16, BF16), (F16, F16)])
@pytest.mark.parametrize("m, n, k, adapters, rank", ADAPTERS)
def test_adapters_tiles(m, n, k, adapters, rank, wt, dtype):
    """Random values, scales and ranks; rows in turns, in runs and without an adapter; what
    lies beyond an adapter's rank, and all of adapter 1, is infinite or NaN."""
    g = generator(m + n + rank)
    a, b = gpu_ints(g, m, k), gpu_ints(g, k, n)
    down = (torch.randn(adapters, rank, k, generator=g, device="cuda") * k ** -0.5).to(wt)
    up = (torch.randn(adapters, n, rank, generator=g, device="cuda") * 0.3).to(wt)
    ranks = torch.randint(0, rank + 1, (adapters,), generator=g, device="cuda").int()
    ranks[0], ranks[-1] = rank, rank + 5
    ids = torch.randint(-1, adapters + 1, (m,), generator=g, device="cuda").int()
    ids[m // 3: m // 2] = 0
    ids[m // 2: m * 3 // 5] = adapters - 1
    ids[-3:] = torch.tensor([0, -1, 1], device="cuda")
    beyond = torch.arange(rank, device="cuda") >= ranks[:, None]
    down.masked_fill_(beyond[:, :, None], float("nan"))
    up.masked_fill_(beyond[:, None, :], INF)
    ranks[1] = rank
    down[1], up[1, ::2], up[1, 1::2] = float("nan"), INF, float("nan")
    sa = (torch.rand(m, generator=g, device="cuda") + 0.5) * 1e-2
    sb = (torch.rand(n, generator=g, device="cuda") + 0.5) * 1e-2
    scaling = torch.rand(adapters, generator=g, device="cuda") + 0.5
    got = ig.adapters_i8(a, b, ids, down, up, sa, sb, ranks=ranks, scaling=scaling,
                         out_dtype=dtype)
    others = torch.where(ids == 1, -1, ids)
    want, base, reach, spread = adapter_terms(a, b, others, down, up, sa, sb, ranks, scaling)
    tiny = {F32: 2.0 ** -150, BF16: 2.0 ** -134, F16: 2.0 ** -25}[dtype]
    bound = (want.abs() * (2 * STEP[F32] + STEP[dtype]) * 1.001 + tiny +
             4 * STEP[F32] * base.abs() + (k + rank + 8) * STEP[F32] * reach +
             2.0 ** -22 * spread)
    keep = ids != 1
    within(got[keep], want[keep], bound[keep])
    assert bool(got[~keep].isnan().all())


@pytest.mark.parametrize("rows, n, k", [(6, 300, 1024), (300, 520, 64), (3000, 2052, 32)])
def test_grouped_rows_that_several_positions_name(rows, n, k):
    """Each element of such a row is one of the positions' values; all positions on one row,
    in pairs on the others' last."""
    g = generator(rows)
    a, b = gpu_ints(g, rows, k), gpu_ints(g, 2, k, n)
    offsets = torch.tensor([0, rows // 3, rows], device="cuda").int()
    order = torch.zeros(rows, device="cuda").int()
    order[rows // 2:] = torch.arange(rows - rows // 2, device="cuda").int() // 2 + 1
    out = torch.full((rows, n), 0.5, device="cuda")
    ig.grouped_i8(a, b, offsets, order, scatter=True, out=out)
    y = torch.cat([a[:rows // 3].double() @ b[0].double(), a[rows // 3:].double() @ b[1].double()])
    assert bool((y[order == 0] == out[0].double()).any(0).all())
    for row in range(1, int(order.max()) + 1):
        assert bool((y[order == row] == out[row].double()).any(0).all())
    assert bool((out[int(order.max()) + 1:] == 0.5).all())


@pytest.mark.parametrize("m, n", [(3, 300), (40, 300), (600, 260)])
@pytest.mark.parametrize("wt", [BF16, F16])
def test_adapters_of_the_largest_rank(m, n, wt):
    rng = np.random.default_rng(m)
    A, B, ids, down, up = make_adapters(rng, m, n, 96, 4, 1024, wt)
    ranks = np.array([1024, 1023, 1009, 1], np.int32)
    check_adapters(A, B, ids, down, up, None, None, ranks, None, F32)


@pytest.mark.parametrize("pad, shift", [(2, 2), (10, 8), (1, 0), (2, 1)])
@pytest.mark.parametrize("wt", [BF16, F16])
def test_adapters_strides_of_large_tiles(pad, shift, wt):
    """`up` with rows and a base at multiples of 4 bytes, which the 256-row tiles take, and
    at others."""
    m, n, k, rank = 4000, 4092, 36, 14
    g = generator(pad)
    a, b = gpu_ints(g, m, k), gpu_ints(g, k, n)
    ids = torch.randint(-1, 7, (m,), generator=g, device="cuda").int()
    down = torch.randn(7, rank, k, generator=g, device="cuda").to(wt)
    up = strided(torch.randn(7, n, rank, generator=g, device="cuda").to(wt), pad, shift)
    one, ranks = torch.ones(m, device="cuda"), torch.full((7,), rank)
    want, base, reach, spread = adapter_terms(a, b, ids, down, up, one, torch.ones(n).cuda(),
                                              ranks, torch.ones(7))
    got = ig.adapters_i8(a, b, ids, strided(down, pad, shift), up, out_dtype=F32)
    within(got, want, want.abs() * 3 * STEP[F32] * 1.001 + 4 * STEP[F32] * base.abs() +
           (k + rank + 8) * STEP[F32] * reach + 2.0 ** -22 * spread)
