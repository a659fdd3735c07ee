"""The operators of include/igemm_rows.h on the GPU against their definitions in
64 bits (rows_reference.py).

Tolerances. A rounding to type T is off by at most eps(T) / 2 of the value (STEP
below; for float16 also half its smallest number). Exact sums take one rounding
into float, one for each scale and one into the output's type. The adapters'
sums are float: a sum of c terms in any order is off by at most c steps of the
sum of its terms' magnitudes, and u goes into the second sum with an error of at
most 2^-22 of its row's largest value."""
import numpy as np
import pytest
import torch

import paper_2302_07594_amd as ig
import rows_reference as ref

pytestmark = pytest.mark.gpu

STEP = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
# half the smallest number of the type (float16 has results below its normal range)
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF = float("inf")


def close(got, want, bound, what=""):
    """bound: an array of how far each value may be from want (float64)."""
    g = got.double().cpu().numpy()
    bad = ~(np.abs(g - want) <= bound)
    if bad.any():
        at = np.argwhere(bad)
        raise AssertionError(f"{what} {len(at)} of {bad.size} out of bounds, first "
                             f"{[(tuple(i), g[tuple(i)], want[tuple(i)]) for i in at[:4]]}")


def rounded(want, dtype, steps):
    """The bound of a value that took `steps` float roundings and one to dtype."""
    return np.abs(want) * (steps * STEP[F32] + STEP[dtype]) * 1.001 + TINY[dtype]


def ints(rng, *shape, lo=-128, hi=127):
    return rng.integers(lo, hi, size=shape, dtype=np.int8, endpoint=True)


def cuda(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def strided(t, pad, shift=0):
    """A copy of t whose rows lie `pad` elements apart more than they are long,
    `shift` elements into its allocation."""
    rows = int(np.prod(t.shape[:-1]))
    ld = t.shape[-1] + pad
    flat = torch.zeros(rows * ld + shift + 64, dtype=t.dtype, device="cuda")
    v = flat[shift:shift + rows * ld].view(*t.shape[:-1], ld)[..., :t.shape[-1]]
    v.copy_(t)
    return v


# ---- route -------------------------------------------------------------------

def check_route(logits, top_k, **kw):
    got = ig.route(logits, top_k, **{k: v.cuda() if k == "bias" and v is not None else v
                                     for k, v in kw.items()})
    want = ref.route(logits.cpu(), top_k, **kw)
    assert np.array_equal(got[0].cpu().numpy(), want[0])
    # (in double, to float once; exp and the sums of double are far below)
    close(got[1], want[1], np.abs(want[1]) * STEP[F32] * 1.01 + TINY[F32], "weights")
    assert np.array_equal(got[2].cpu().numpy(), want[2])
    assert np.array_equal(got[3].cpu().numpy(), want[3])
    return got


@pytest.mark.parametrize("tokens, experts, top_k, groups, top_groups, group_best", [
    (1, 1, 1, 1, 1, 1), (1, 4, 4, 1, 1, 1), (3, 7, 3, 1, 1, 2), (8, 64, 8, 1, 1, 1),
    (65, 65, 8, 5, 2, 1), (33, 128, 8, 8, 4, 2), (100, 256, 8, 8, 4, 2), (17, 250, 64, 2, 2, 2),
    (5, 512, 16, 64, 7, 1), (3, 1024, 1, 4, 1, 2), (2, 1000, 33, 1, 1, 1), (9, 64, 20, 64, 20, 2),
    (300, 16, 2, 4, 3, 1), (1025, 60, 4, 1, 1, 1), (4099, 160, 6, 8, 3, 1)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias, dtype", [(False, F32), (True, F32), (True, BF16), (False, F16)])
def test_route(tokens, experts, top_k, groups, top_groups, group_best, score, bias, dtype):
    g = torch.Generator().manual_seed(tokens * 1009 + experts)
    x = (torch.randn(tokens, experts, generator=g) * 2).to(dtype)
    b = torch.randn(experts, generator=g) * 0.2 if bias else None
    check_route(x.cuda(), top_k, bias=b, groups=groups, top_groups=top_groups,
                group_best=group_best, score=score, renormalise=top_k % 2 == 0, scale=1.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
def test_route_ties_and_masks(score, bias):
    """Equal keys, masked experts, rows that have few or none left, infinities,
    NaN, the type's lowest value, logits that exp and the sigmoid flatten."""
    E = 70
    x = torch.zeros(16, E)
    x[1] = -INF
    x[2, 5:] = -INF
    x[3] = float("nan")
    x[4, ::2] = torch.finfo(F32).min
    x[5] = torch.finfo(F32).min
    x[6, 10] = INF
    x[7, 10], x[7, 60] = INF, INF
    x[8] = torch.arange(E) // 7
    x[9] = -torch.arange(E).float() * 40
    x[10] = 60.0 + torch.arange(E)
    x[11, 3], x[11, 4] = -INF, float("nan")
    x[12] = torch.arange(E) % 2
    x[13] = -300.0
    x[14, 69] = 1e-30
    b = torch.zeros(E) if bias else None
    check_route(x.cuda(), 8, bias=b, score=score)
    check_route(x.cuda(), 8, bias=b, score=score, groups=10, top_groups=3, group_best=2,
                renormalise=False)
    check_route(x.cuda(), 3, bias=b, score=score, groups=7, top_groups=1)


def test_route_biases_that_exclude():
    x = torch.zeros(3, 12)
    b = torch.zeros(12)
    b[0], b[3], b[5], b[7] = -INF, float("nan"), INF, -1e30
    check_route(x.cuda(), 12, bias=b)
    check_route(x.cuda(), 4, bias=b, groups=4, top_groups=2, group_best=2)


@pytest.mark.parametrize("pad, shift", [(0, 1), (3, 0), (5, 3), (64, 0)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_route_strides(pad, shift, dtype):
    x = torch.randn(37, 100).to(dtype)
    check_route(strided(x, pad, shift), 5, groups=4, top_groups=2)


def test_route_without_plan_and_without_tokens():
    x = torch.randn(9, 20).cuda()
    ids, w, off, order = ig.route(x, 3, plan=False)
    assert off is None and order is None
    want = ref.route(x.cpu(), 3)
    assert np.array_equal(ids.cpu().numpy(), want[0])
    ids, w, off, order = ig.route(x[:0], 3)
    assert ids.shape == (0, 3) and order.shape == (0,) and off.cpu().tolist() == [0] * 21


@pytest.mark.parametrize("tokens, experts, top_k", [(20000, 8, 2), (3000, 1024, 8), (7000, 64, 1)])
def test_route_long_and_uneven_plans(tokens, experts, top_k):
    """Plans of many slots, nearly all of one expert, or none of some."""
    g = torch.Generator().manual_seed(5)
    x = torch.randn(tokens, experts, generator=g)
    x[:, 3] += 6.0
    x[: tokens // 3] = -INF
    check_route(x.cuda(), top_k)


# ---- the experts' products -----------------------------------------------------

def check_grouped(A, B, offsets, order, sa, sb, slots, scatter, rows, out_rows, dtype, pads=None,
                  **kw):
    want = np.full((out_rows, B.shape[2]), 7.0)
    want, wrote = ref.grouped(A, B, offsets, order, sa, sb, slots, scatter, rows, want)
    a, b = cuda(A), cuda(B)
    out = torch.full((out_rows, B.shape[2]), 7.0, dtype=dtype, device="cuda")
    if pads:
        pa, pb, po, shift = pads
        a, b, out = strided(a, pa, shift), strided(b, pb, shift), strided(out, po, shift)
    got = ig.grouped_i8(a, b, cuda(np.asarray(offsets, np.int32)),
                        cuda(None if order is None else np.asarray(order, np.int32)),
                        scale_a=cuda(sa), scale_b=cuda(sb), slots=slots, scatter=scatter,
                        rows=rows, out=out, **kw)
    assert got is out
    if out.numel():
        close(got[~torch.from_numpy(wrote).cuda()], want[~wrote], 0.0, "rows left alone")
        close(got[torch.from_numpy(wrote).cuda()], want[wrote], rounded(want[wrote], dtype, 3))
        if pads and pads[2]:   # what lies between the rows of out
            whole = out.as_strided((out_rows, out.stride(0)), (out.stride(0), 1),
                                   out.storage_offset())
            assert not whole[:, B.shape[2]:].any()


def split(rng, rows, groups, first=0, last=0):
    """Ascending offsets with empty groups among them."""
    cuts = np.sort(rng.integers(first, rows - last, size=groups - 1, endpoint=True))
    return np.concatenate([[first], cuts, [rows - last]]).astype(np.int32)


SIZES = [(1, 1, 1, 1), (1, 130, 64, 3), (7, 16, 15, 2), (40, 33, 17, 5), (64, 256, 128, 4),
         (65, 100, 100, 9), (129, 257, 130, 3), (300, 64, 1000, 70), (500, 384, 256, 2),
         (1000, 17, 63, 7), (33, 1025, 511, 4), (16, 4096, 256, 8), (260, 128, 2048, 1)]


@pytest.mark.parametrize("rows, n, k, groups", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_grouped(rows, n, k, groups, dtype):
    rng = np.random.default_rng(rows * 31 + n)
    A, B = ints(rng, rows, k), ints(rng, groups, k, n)
    sa = rng.random(rows, dtype=np.float32) * 1e-3
    sb = rng.random((groups, n), dtype=np.float32) * 1e-2
    check_grouped(A, B, split(rng, rows, groups), None, sa, sb, 0, False, rows, rows, dtype)


@pytest.mark.parametrize("pads", [(1, 0, 0, 0), (0, 3, 0, 0), (4, 4, 1, 4), (12, 4, 7, 8),
                                  (5, 9, 3, 1), (0, 0, 0, 2), (16, 16, 16, 16)])
@pytest.mark.parametrize("rows, n, k, groups", [(1, 130, 64, 3), (70, 64, 128, 4),
                                                (150, 129, 193, 3), (9, 48, 256, 2)])
def test_grouped_strides(rows, n, k, groups, pads):
    rng = np.random.default_rng(n + k)
    A, B = ints(rng, rows, k), ints(rng, groups, k, n)
    check_grouped(A, B, split(rng, rows, groups), None, None, None, 0, False, rows, rows, F32,
                  pads)


@pytest.mark.parametrize("tokens, top_k, groups, n, k", [(1, 1, 1, 16, 64), (1, 8, 32, 128, 256),
                                                         (5, 3, 8, 70, 129), (90, 4, 6, 200, 192),
                                                         (333, 2, 5, 96, 80)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_grouped_gathers_and_scatters(tokens, top_k, groups, n, k, dtype):
    rng = np.random.default_rng(tokens)
    rows = tokens * top_k
    ids = rng.integers(0, groups, size=rows)
    order = np.argsort(ids, kind="stable").astype(np.int32)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(ids, minlength=groups))])
    B = ints(rng, groups, k, n)
    sb = rng.random((groups, n), dtype=np.float32)
    sa = rng.random(tokens, dtype=np.float32)
    check_grouped(ints(rng, tokens, k), B, offsets, order, sa, sb, top_k, False, rows, rows, dtype)
    sa = rng.random(rows, dtype=np.float32)
    check_grouped(ints(rng, rows, k), B, offsets, order, sa, sb, 0, True, rows, rows, dtype)
    check_grouped(ints(rng, tokens, k), B, offsets, order, None, sb, top_k, True, rows, rows + 3,
                  dtype)


@pytest.mark.parametrize("rows", [5, 90])
def test_grouped_plans_that_leave_rows_out(rows):
    """Offsets that begin late, end early, pass the rows or fall back; orders
    with -1, entries past the rows of A and out, and the same slot twice."""
    rng = np.random.default_rng(3)
    n, k = 70, 96
    A, B = ints(rng, rows, k), ints(rng, 4, k, n)
    for offsets in ([0, 0, 0, 0, 0], [2, 2, 3, rows - 1, rows - 1], [-5, 1, 2, 3, 4],
                    [0, 1, 2, 3, rows + 1000], [rows + 7] * 5,
                    [0, 2 ** 31 - 1, 3, 3, 3], [-2 ** 31, 0, 0, 0, rows]):
        check_grouped(A, B, offsets, None, None, None, 0, False, rows, rows, F32)
    order = rng.permutation(rows)
    order[0], order[1], order[2], order[3] = -1, rows, 2 ** 31 - 1, -2 ** 31
    for slots, scatter in ((0, False), (0, True), (1, False), (1, True), (3, False)):
        check_grouped(A, B, [0, 2, 3, 4, rows], order, None, None, slots, scatter, rows, rows, F32)
    check_grouped(A, B, [0, 2, 3, 4, rows], order, None, None, 1, True, rows, rows - 2, F32)
    same = np.zeros(rows, np.int32)     # every position the same token
    check_grouped(A, B, [0, 2, 3, 4, rows], same, None, None, 1, False, rows, rows, F32)


def test_grouped_extremes():
    """Sums at the ends of int32, k = 0, B's groups at stride 0, rows of out
    beyond the positions."""
    k = 131071
    A = np.full((3, k), -128, np.int8)
    A[1] = 127
    B = np.full((2, k, 5), -128, np.int8)
    check_grouped(A, B, [0, 2, 3], None, None, None, 0, False, 3, 3, F32)
    out = torch.full((4, 6), 7.0, device="cuda")
    ig.grouped_i8(torch.zeros(3, 0, dtype=torch.int8, device="cuda"),
                  torch.zeros(2, 0, 6, dtype=torch.int8, device="cuda"),
                  torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda"), out=out)
    assert out.cpu().tolist() == [[0.0] * 6] * 3 + [[7.0] * 6]
    rng = np.random.default_rng(0)
    A, B = ints(rng, 9, 64), ints(rng, 1, 64, 32)
    shared = cuda(B).expand(3, 64, 32)
    got = ig.grouped_i8(cuda(A), shared, torch.tensor([0, 4, 4, 9], dtype=torch.int32).cuda(),
                        out_dtype=F32)
    assert np.array_equal(got.cpu().numpy().astype(np.int64),
                          A.astype(np.int64) @ B[0].astype(np.int64))


def test_grouped_far_weights():
    """The last group's weights lie past 4 GiB."""
    n, k, groups = 64, 64, 3
    stride = 3 << 30
    flat = torch.empty((groups - 1) * stride + k * n, dtype=torch.int8, device="cuda")
    rng = np.random.default_rng(1)
    A, B = ints(rng, 20, k), ints(rng, groups, k, n)
    b = flat.as_strided((groups, k, n), (stride, n, 1))
    b.copy_(cuda(B))
    got = ig.grouped_i8(cuda(A), b, torch.tensor([0, 6, 7, 20], dtype=torch.int32).cuda(),
                        out_dtype=F32)
    want, _ = ref.grouped(A, B, [0, 6, 7, 20], None, None, None, 0, False, 20, np.zeros((20, n)))
    assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("rows", [700, 6])
def test_grouped_far_output(rows):
    """Rows of out past 4 GiB, gathered from one row and scattered in turned order."""
    n, ld = 48, 1 << 22 if rows > 6 else (1 << 22) - 3
    flat = torch.zeros((rows - 1) * ld + n, dtype=BF16, device="cuda")
    out = flat.as_strided((rows, n), (ld, 1))
    order = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device="cuda")
    a = torch.arange(rows, device="cuda").remainder(100).to(torch.int8)[:, None].contiguous()
    b = torch.ones(1, 1, n, dtype=torch.int8, device="cuda")
    ig.grouped_i8(a, b, torch.tensor([0, rows], dtype=torch.int32).cuda(), order, slots=1,
                  scatter=True, out=out)
    assert torch.equal(out, a.to(BF16).expand(rows, n))


# ---- the sum of a token's slots -------------------------------------------------

@pytest.mark.parametrize("tokens, top_k, n", [(1, 1, 1), (1, 8, 4096), (7, 3, 33), (130, 2, 1000),
                                              (3, 70, 17), (1000, 4, 64), (5, 8, 8200)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("pads", [(0, 0, 0), (1, 3, 5), (8, 8, 8)])
def test_combine(tokens, top_k, n, dtype, pads):
    g = torch.Generator().manual_seed(n)
    Z = torch.randn(tokens * top_k, n, generator=g).to(dtype)
    w = torch.randn(tokens, top_k, generator=g)
    ids = torch.where(torch.rand(tokens, top_k, generator=g) < 0.3, -1, 2).int()
    # what an empty slot holds never matters
    empty = ids.flatten() < 0
    Z[empty] = float("nan")
    w[ids < 0] = INF
    base = torch.randn(tokens, n, generator=g).to(dtype)
    z64 = torch.where(empty[:, None], 0.0, Z.double()).view(tokens, top_k, n)
    w64 = torch.where(ids < 0, 0.0, w.double())[:, :, None]
    part, size = (z64 * w64).sum(1), (z64 * w64).abs().sum(1)
    put = [strided(t.cuda(), p) for t, p in zip((Z, base, torch.zeros(tokens, n, dtype=dtype)),
                                                pads)]
    for b in (None, put[1]):
        want = part if b is None else part + base.double()
        size_b = size if b is None else size + base.double().abs()
        bound = (top_k + 2) * STEP[F32] * size_b + STEP[dtype] * want.abs() * 1.001 + TINY[dtype]
        got = ig.combine(put[0], w.cuda(), ids=ids.cuda(), base=b, out=put[2])
        assert got is put[2]
        close(got, want.numpy(), bound.numpy())
    close(ig.combine(put[0], w.cuda(), ids=ids.cuda(), base=put[1], out=put[1]), want.numpy(),
          bound.numpy(), "in place")
    full = torch.randn(tokens * top_k, n, generator=g).to(dtype)
    wf = torch.randn(tokens, top_k, generator=g)
    terms = full.double().view(tokens, top_k, n) * wf.double()[:, :, None]
    close(ig.combine(full.cuda(), wf.cuda()), terms.sum(1).numpy(),
          ((top_k + 2) * STEP[F32] * terms.abs().sum(1) +
           STEP[dtype] * terms.sum(1).abs() * 1.001 + TINY[dtype]).numpy())


# ---- adapters --------------------------------------------------------------------

def test_combine_far_rows():
    """Rows of Z, base and out past 4 GiB."""
    n, ld = 40, (1 << 31) + 8
    flat = torch.empty(3 * ld + 3 * n, dtype=BF16, device="cuda")
    Z = flat.as_strided((4, n), (ld, 1))
    base = flat.as_strided((2, n), (ld, 1), n)
    out = flat.as_strided((2, n), (ld, 1), 2 * n)
    Z.copy_(torch.arange(4, device="cuda")[:, None].expand(4, n))
    base.fill_(8)
    w = torch.tensor([[1.0, 2.0], [4.0, 8.0]], device="cuda")
    got = ig.combine(Z, w, base=base, out=out)
    assert torch.equal(got.float(), torch.tensor([[10.0], [40.0]], device="cuda").expand(2, n))


def make_adapters(rng, m, n, k, adapters, rank, wt, every=None):
    A, B = ints(rng, m, k), ints(rng, k, n)
    down = (torch.from_numpy(rng.standard_normal((adapters, rank, k))) * k ** -0.5).to(wt)
    up = (torch.from_numpy(rng.standard_normal((adapters, n, rank))) * 0.3).to(wt)
    ids = rng.integers(-1, adapters, size=m).astype(np.int32) if every is None else \
        np.asarray(every, np.int32)
    return A, B, ids, down, up


def check_adapters(A, B, ids, down, up, sa, sb, ranks, scaling, dtype, pads=None, **kw):
    d64 = None if down is None else down.double().numpy()
    u64 = None if up is None else up.double().numpy()
    want, base, reach, spread = ref.adapters(A, B, sa, sb, ids, d64, u64, ranks, scaling)
    a, b = cuda(A), cuda(B)
    d, u = (None if t is None else t.cuda() for t in (down, up))
    out = torch.full(want.shape, 7.0, dtype=dtype, device="cuda")
    if pads:
        pa, pb, pd, pu, po, shift = pads
        a, b, d, u, out = (strided(t, p, shift) for t, p in
                           zip((a, b, d, u, out), (pa, pb, pd, pu, po)))
    got = ig.adapters_i8(a, b, cuda(ids), d, u, scale_a=cuda(sa), scale_b=cuda(sb),
                         ranks=cuda(ranks), scaling=cuda(scaling), out=out, **kw)
    assert got is out
    terms = A.shape[1] + (0 if up is None else up.shape[2]) + 8
    bound = (rounded(want, dtype, 2) + 4 * STEP[F32] * np.abs(base) +
             terms * STEP[F32] * reach + 2.0 ** -22 * spread)
    close(got, want, bound)


@pytest.mark.parametrize("m, n, k, adapters, rank", [
    (1, 1, 1, 1, 1), (1, 64, 64, 2, 8), (3, 33, 17, 2, 3), (16, 256, 256, 16, 16),
    (17, 100, 100, 5, 17), (64, 130, 192, 3, 64), (40, 128, 128, 40, 4), (129, 65, 300, 7, 128),
    (300, 200, 64, 2, 24), (33, 48, 1000, 9, 200), (8, 1024, 512, 3, 32), (260, 384, 128, 4, 16)])
@pytest.mark.parametrize("dtype, wt", [(F32, BF16), (F32, F16), (BF16, BF16), (F16, F16)])
def test_adapters(m, n, k, adapters, rank, dtype, wt):
    rng = np.random.default_rng(m * 7 + n)
    A, B, ids, down, up = make_adapters(rng, m, n, k, adapters, rank, wt)
    sa = (rng.random(m, dtype=np.float32) + 0.5) * 1e-2
    sb = (rng.random(n, dtype=np.float32) + 0.5) * 1e-3
    scaling = rng.random(adapters, dtype=np.float32) + 0.5
    check_adapters(A, B, ids, down, up, sa, sb, None, scaling, dtype)


@pytest.mark.parametrize("layout", ["runs", "turns", "none", "one", "outside"])
@pytest.mark.parametrize("m", [5, 150])
def test_adapters_which_rows_have_them(layout, m):
    rng = np.random.default_rng(11)
    n = {"runs": 6, "turns": 6, "none": 2, "one": 1, "outside": 4}[layout]
    every = {"runs": np.arange(m) * n // m, "turns": np.arange(m) % n - 1,
             "none": np.full(m, -1), "one": np.zeros(m),
             "outside": np.where(np.arange(m) % 3 == 0, 2 ** 31 - 1, np.arange(m) % 8 - 3)}[layout]
    A, B, ids, down, up = make_adapters(rng, m, 140, 160, n, 16, BF16, every)
    check_adapters(A, B, ids, down, up, None, None, None, None, F32)


def test_adapters_ranks():
    """Each adapter its own rank; what lies beyond holds infinities and NaN."""
    rng = np.random.default_rng(12)
    A, B, ids, down, up = make_adapters(rng, 90, 70, 100, 6, 20, F16)
    ranks = np.array([0, 1, 7, 20, 99, -3], np.int32)
    for a, r in enumerate(np.clip(ranks, 0, 20)):
        down[a, r:] = float("nan")
        up[a, :, r:] = INF
    check_adapters(A, B, ids, down, up, None, None, ranks, None, F32)


@pytest.mark.parametrize("bad", [float("nan"), INF])
@pytest.mark.parametrize("wt", [BF16, F16])
def test_adapters_keep_to_their_rows(bad, wt):
    """An adapter full of infinities or NaN spoils its own rows alone."""
    rng = np.random.default_rng(13)
    A, B, ids, down, up = make_adapters(rng, 70, 90, 130, 4, 12, wt, np.arange(70) % 5 - 1)
    down[2], up[2] = bad, bad
    out = ig.adapters_i8(cuda(A), cuda(B), cuda(ids), down.cuda(), up.cuda(), out_dtype=F32)
    keep = ids != 2
    want, base, reach, spread = ref.adapters(A, B, None, None, np.where(keep, ids, -1),
                                             down.double().numpy(), up.double().numpy(), None,
                                             None)
    bound = rounded(want, F32, 4) + 4 * STEP[F32] * np.abs(base) + 200 * STEP[F32] * reach + \
        2.0 ** -22 * spread
    close(out[torch.from_numpy(keep).cuda()], want[keep], bound[keep])
    assert not out[torch.from_numpy(~keep).cuda()].isfinite().any()


@pytest.mark.parametrize("pads", [(1, 3, 1, 1, 5, 1), (4, 4, 4, 4, 4, 4), (16, 16, 8, 8, 8, 0),
                                  (0, 0, 3, 5, 0, 0)])
@pytest.mark.parametrize("m, n, k, rank", [(2, 64, 64, 16), (100, 72, 136, 9)])
def test_adapters_strides(m, n, k, rank, pads):
    rng = np.random.default_rng(14)
    A, B, ids, down, up = make_adapters(rng, m, n, k, 3, rank, BF16)
    check_adapters(A, B, ids, down, up, None, None, None, None, F32, pads)


def test_adapters_wide_range_of_values():
    """u over forty orders of two, float16 and bfloat16 weights."""
    rng = np.random.default_rng(15)
    for wt in (F16, BF16):
        A, B, ids, down, up = make_adapters(rng, 40, 64, 128, 3, 16, wt)
        down = (down.float() * torch.exp2(-torch.arange(16).float())[None, :, None]).to(wt)
        for scale in (2.0 ** -40, 1.0, 2.0 ** 40):
            sa = np.full(40, scale, np.float32)
            check_adapters(A, B, ids, down, up, sa, None, None, None, F32)


@pytest.mark.parametrize("wt", [BF16, F16])
@pytest.mark.parametrize("k", [9, 500, 512, 513, 1024, 1100, 1536, 2048, 2059, 2560])
def test_adapters_lengths(k, wt):
    """Tiles of 512 k in u's product: none to five whole ones, with and without a rest; 16
    and 33 ranks, more adapters than one workgroup of a block takes."""
    rng = np.random.default_rng(k)
    for m, rank, adapters in ((300, 16, 3), (140, 33, 40)):
        A, B, ids, down, up = make_adapters(rng, m, 40, k, adapters, rank, wt)
        check_adapters(A, B, ids, down, up, None, None, None, None, F32)


@pytest.mark.parametrize("m, n", [(3, 64), (400, 512), (8192, 2048)])
def test_adapters_far_matrices(m, n):
    """The second adapter's matrices lie past 4 GiB: few rows, the 128-row tiles, the
    256-row ones. Sums of ones, exact in every type."""
    k, rank, far = 64, 16, 5 << 29
    down = torch.zeros(far + rank * k, dtype=BF16, device="cuda").as_strided(
        (2, rank, k), (far, k, 1))
    up = torch.zeros(far + n * rank, dtype=BF16, device="cuda").as_strided(
        (2, n, rank), (far, rank, 1))
    down[1] = 1
    up[0] = up[1] = 1
    a = torch.ones(m, k, dtype=torch.int8, device="cuda")
    ids = torch.arange(m, dtype=torch.int32, device="cuda") % 3  # (2: none)
    got = ig.adapters_i8(a, torch.ones(k, n, dtype=torch.int8, device="cuda"), ids, down, up,
                         out_dtype=F32)
    want = torch.where(ids == 1, float(k + k * rank), float(k))[:, None].expand(m, n)
    assert torch.equal(got, want)


@pytest.mark.parametrize("wt", [BF16, F16])
@pytest.mark.parametrize("m, n", [(3, 40), (100, 300), (4096, 4096)])
def test_adapters_of_the_largest_floats(m, n, wt):
    """u within half a bf16 step of the largest float, which bf16 would round to infinity."""
    u, v = float(np.float32(3.4e38)), 2.0 ** -20
    a = torch.ones(m, 1, dtype=torch.int8, device="cuda")
    b = torch.zeros(1, n, dtype=torch.int8, device="cuda")
    ids = torch.zeros(m, dtype=torch.int32, device="cuda")
    down = torch.ones(1, 1, 1, dtype=wt, device="cuda")
    up = torch.full((1, n, 1), v, dtype=wt, device="cuda")
    got = ig.adapters_i8(a, b, ids, down, up, scaling=torch.full((1,), u, device="cuda"),
                         out_dtype=F32)
    assert bool((got == u * v).all())


def test_projection_without_adapters():
    rng = np.random.default_rng(16)
    for m, n, k in ((1, 4096, 512), (37, 129, 77), (200, 256, 256)):
        A, B = ints(rng, m, k), ints(rng, k, n)
        sa, sb = rng.random(m, dtype=np.float32), rng.random(n, dtype=np.float32)
        check_adapters(A, B, None, None, None, sa, sb, None, None, BF16)
        # no adapters, or adapters of rank 0
        for adapters, rank in ((0, 8), (3, 0)):
            down = torch.zeros(adapters, rank, k, dtype=BF16)
            up = torch.zeros(adapters, n, rank, dtype=BF16)
            check_adapters(A, B, np.zeros(m, np.int32), down, up, sa, sb, None, None, F32)
    out = ig.adapters_i8(torch.zeros(3, 0, dtype=torch.int8, device="cuda"),
                         torch.zeros(0, 5, dtype=torch.int8, device="cuda"), out_dtype=F32)
    assert out.cpu().tolist() == [[0.0] * 5] * 3


# ---- together, and how they are called -------------------------------------------

def quantise(x):
    """int8 rows and their scales (a symmetric quantisation)."""
    s = x.float().abs().amax(dim=1).clamp_min(1e-6) / 127
    return torch.round(x.float() / s[:, None]).to(torch.int8), s


class Layer:
    """A sparse feed-forward layer beside an adapted projection, as a decoder
    runs it: route, first product, gate, second product, sum."""

    def __init__(self, tokens, d=192, f=128, experts=9, top_k=3, seed=21):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        i = lambda *s: torch.empty(*s, dtype=torch.int8, device="cuda").random_(  # noqa: E731
            -127, 128, generator=g)
        self.top_k, self.f, self.x, self.gate = top_k, f, r(tokens, d), r(d, experts)
        self.x[tokens // 2] = 0.0
        self.w1, self.w2, self.w0 = i(experts, d, 2 * f), i(experts, f, d), i(d, d)
        self.s1, self.s2 = (torch.rand(experts, n, generator=g, device="cuda") * 1e-3
                            for n in (2 * f, d))
        self.s0 = torch.rand(d, generator=g, device="cuda") * 1e-3
        self.ids = (torch.arange(tokens, device="cuda") % 4 - 1).int()
        self.down, self.up = r(3, 8, d).bfloat16(), r(3, d, 8).bfloat16()

    def __call__(self, keep=None, **kw):
        x, s = quantise(self.x)
        logits = self.x @ self.gate
        logits[3 % len(logits)] = -INF        # a padded token
        ids, w, offsets, order = ig.route(logits, self.top_k, **kw)
        h = ig.grouped_i8(x, self.w1, offsets, order, scale_a=s, scale_b=self.s1,
                          slots=self.top_k, **kw)
        h32 = h.float()
        a, sa = quantise(torch.nn.functional.silu(h32[:, :self.f]) * h32[:, self.f:])
        z = ig.grouped_i8(a, self.w2, offsets, order, scale_a=sa, scale_b=self.s2, scatter=True,
                          **kw)
        base = ig.adapters_i8(x, self.w0, self.ids, self.down, self.up, scale_a=s,
                              scale_b=self.s0, **kw)
        out = ig.combine(z, w, ids=ids, base=base, **kw)
        if keep is not None:
            keep.update(x=x, s=s, logits=logits, ids=ids, w=w, offsets=offsets, order=order, h=h,
                        a=a, sa=sa, z=z, base=base)
        return out


@pytest.mark.parametrize("tokens", [1, 5, 130])
def test_layer(tokens):
    """Each step against its definition on what the step before it gave."""
    layer, k = Layer(tokens), {}
    out = layer(keep=k)
    n = lambda t: t.cpu().numpy()  # noqa: E731
    ids, w, offsets, order = ref.route(k["logits"].cpu(), layer.top_k)
    assert np.array_equal(n(k["ids"]), ids) and np.array_equal(n(k["order"]), order)
    rows = tokens * layer.top_k
    want, _ = ref.grouped(n(k["x"]), n(layer.w1), offsets, order, n(k["s"]), n(layer.s1),
                          layer.top_k, False, rows, np.zeros((rows, 2 * layer.f)))
    close(k["h"], want, rounded(want, BF16, 3))
    want, _ = ref.grouped(n(k["a"]), n(layer.w2), offsets, order, n(k["sa"]), n(layer.s2), 0,
                          True, rows, np.zeros((rows, 192)))
    close(k["z"], want, rounded(want, BF16, 3))
    want, base, reach, spread = ref.adapters(
        n(k["x"]), n(layer.w0), n(k["s"]), n(layer.s0), n(layer.ids),
        layer.down.double().cpu().numpy(), layer.up.double().cpu().numpy(), None, None)
    close(k["base"], want, rounded(want, BF16, 2) + 4 * STEP[F32] * np.abs(base) +
          208 * STEP[F32] * reach + 2.0 ** -22 * spread)
    z = k["z"].double().cpu().numpy().reshape(tokens, layer.top_k, -1) * n(k["w"])[:, :, None]
    b = k["base"].double().cpu().numpy()
    want = z.sum(1) + b
    close(out, want, rounded(want, BF16, 0) +
          (layer.top_k + 2) * STEP[F32] * (np.abs(z).sum(1) + np.abs(b)))


def test_layer_on_a_stream_and_again():
    """The same bits on another stream (a torch one, or its handle) and on a
    second run."""
    layer = Layer(70)
    want = layer()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for s in (side, int(side.cuda_stream), None):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = layer(stream=s)
        side.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("tokens", [1, 8, 200])
def test_layer_captured_and_replayed(tokens):
    layer = Layer(tokens)
    other = Layer(tokens, seed=22)
    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer()
    first = layer.x.clone()
    for x in (first, other.x, first * 0.5, other.x):
        layer.x.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = layer()            # eager work between the replays
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_two_graphs_that_share_a_workspace():
    """Two captured calls on one workspace, replayed in turn on one stream."""
    rng = np.random.default_rng(30)
    ws = torch.empty(16 << 20, dtype=torch.uint8, device="cuda")
    calls = []
    for m, n, k in ((8, 512, 512), (40, 256, 1024)):
        A, B, ids, down, up = make_adapters(rng, m, n, k, 3, 16, BF16)
        args = [cuda(A), cuda(B), cuda(ids), down.cuda(), up.cuda()]
        out = torch.zeros(m, n, device="cuda")
        ig.adapters_i8(*args, out=out, workspace=ws)
        torch.cuda.synchronize()
        want = out.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ig.adapters_i8(*args, out=out, workspace=ws)
        calls.append((graph, args, out, want))
    for _ in range(3):
        for graph, _, out, want in calls:
            out.zero_()
            ws.fill_(0xff)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_workspaces():
    x = torch.zeros(4, 64, dtype=torch.int8, device="cuda")
    w = torch.zeros(64, 32, dtype=torch.int8, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    down = torch.zeros(1, 8, 64, dtype=BF16, device="cuda")
    up = torch.zeros(1, 32, 8, dtype=BF16, device="cuda")
    small = torch.zeros(16, dtype=torch.uint8, device="cuda")
    with pytest.raises(ig.IgemmError) as e:
        ig.adapters_i8(x, w, ids, down, up, workspace=small)
    assert e.value.status == ig.IGEMM_ENOMEM
    big = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    with pytest.raises(ig.IgemmError) as e:
        ig.adapters_i8(x, w, ids, down, up, workspace=big[16:])
    assert e.value.status == ig.IGEMM_EINVAL
    big.fill_(0xff)
    assert not ig.adapters_i8(x, w, ids, down, up, workspace=big).any()


def test_refusals_leave_the_output_alone():
    a = torch.zeros(4, 64, dtype=torch.int8, device="cuda")
    b = torch.zeros(2, 64, 32, dtype=torch.int8, device="cuda")
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    out = torch.full((4, 32), 7.0, device="cuda")
    for bad in (dict(offsets=off[:2]), dict(offsets=off.long()), dict(A=a.t()),
                dict(B=b.transpose(1, 2)), dict(out=out[:, ::2]), dict(scale_a=off),
                dict(order=off.cpu()), dict(out_dtype=BF16), dict(rows=-1), dict(slots=-1)):
        kw = dict(A=a, B=b, offsets=off, out=out) | bad
        with pytest.raises((TypeError, ValueError, ig.IgemmError)):
            ig.grouped_i8(**kw)
    with pytest.raises(TypeError):
        ig.route(torch.zeros(2, 4, device="cuda"), 2, stream="0")
    with pytest.raises(ValueError):
        ig.route(torch.zeros(2, 4, device="cuda"), 2, score="relu")
    with pytest.raises(ig.IgemmError):
        ig.route(torch.zeros(2, 4, device="cuda"), 5)
    torch.cuda.synchronize()
    assert bool((out == 7).all())


def test_no_gradient_is_dropped_in_silence():
    """A float operand whose gradient would be wanted is refused, and taken where none
    is recorded."""
    layer = Layer(8)
    k = {}
    layer(keep=k)
    a, y = k["x"], torch.empty(8, 192, dtype=BF16, device="cuda")
    out = torch.zeros(24, 256, dtype=BF16, device="cuda")
    sa = k["s"]
    calls = [
        ("logits", lambda t: ig.route(t, 3)[1], k["logits"]),
        ("scale_a", lambda t: ig.grouped_i8(a, layer.w1, k["offsets"], k["order"], t, slots=3,
                                            out=out), sa),
        ("Z", lambda t: ig.combine(t, k["w"], out=y), k["z"]),
        ("weights", lambda t: ig.combine(k["z"], t, out=y), k["w"]),
        ("down", lambda t: ig.adapters_i8(a, layer.w0, layer.ids, t, layer.up, out=y), layer.down),
        ("up", lambda t: ig.adapters_i8(a, layer.w0, layer.ids, layer.down, t, out=y), layer.up)]
    for name, call, t in calls:
        want = call(t).clone()
        leaf = t.detach().clone().requires_grad_()
        with pytest.raises(ValueError, match=f"detach {name}"):
            call(leaf)
        with torch.no_grad():
            assert torch.equal(call(leaf), want), name


def test_offsets_that_do_not_ascend_stay_inside():
    """The values are not specified, but nothing beside out is written: here the tiles of
    the groups together are 2^31 and more."""
    rows, groups = 1 << 22, 65536
    a = torch.ones(rows, 1, dtype=torch.int8, device="cuda")
    b = torch.ones(groups, 1, 1, dtype=torch.int8, device="cuda")
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda").repeat(groups // 2)
    off = torch.cat([off, off[:1]])
    whole = torch.full((rows + 128, 1), 7.0, device="cuda")
    out = whole[64:-64]
    ig.grouped_i8(a, b, off, out=out)
    torch.cuda.synchronize()
    assert bool((whole[:64] == 7).all()) and bool((whole[-64:] == 7).all())
    assert bool(((out == 1) | (out == 7)).all())


def test_plain_calls_take_the_compiled_binding(monkeypatch):
    """What the Python code would do is the same, and plain calls do not reach it."""
    layer = Layer(40)
    k = {}
    layer(keep=k)
    a, off, order = k["x"], k["offsets"], k["order"]
    out = torch.zeros(120, 256, dtype=BF16, device="cuda")  # (the padded token has no rows)
    y = torch.empty(40, 192, dtype=BF16, device="cuda")
    calls = [
        lambda **kw: ig.route(k["logits"], 3, **kw),
        lambda **kw: ig.grouped_i8(a, layer.w1, off, order, k["s"], layer.s1, slots=3, out=out,
                                   **kw),
        lambda **kw: ig.combine(k["z"], k["w"], ids=k["ids"], base=k["base"], out=y, **kw),
        lambda **kw: ig.adapters_i8(a, layer.w0, layer.ids, layer.down, layer.up, k["s"],
                                    layer.s0, out=y, **kw)]
    copy = lambda r: tuple(t.clone() for t in (r if isinstance(r, tuple) else (r,)))  # noqa: E731
    slow = [copy(f(stream=torch.cuda.current_stream())) for f in calls]

    def refuse(*a, **kw):
        raise AssertionError("the Python path ran")
    monkeypatch.setattr(ig, "_on", refuse)
    for f, want in zip(calls, slow):
        assert all(torch.equal(g, w) for g, w in zip(copy(f()), want))
    with pytest.raises(ig.IgemmError):
        ig.route(k["logits"], 10)
