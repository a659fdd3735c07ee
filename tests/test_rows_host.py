"""Host-side checks of include/igemm_rows.h (no GPU): the exports, the
refusals before any HIP call, calls with nothing to do, the workspace queries
and the reference that the GPU tests compare with."""
import contextlib
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2302_07594_amd as ig
import rows_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, Q, R, S = 0x10000, 0x20000, 0x30000, 0x40000  # never dereferenced
E, N = ig.IGEMM_EINVAL, ig.IGEMM_ENOTSUP


def declared():
    text = open(os.path.join(ROOT, "include", "igemm_rows.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"^\s*int\s+(igemm_\w+)\s*\(", text, re.M)))


def test_library_exports_every_declared_symbol():
    names = declared()
    assert names == ["igemm_combine", "igemm_i8_adapters", "igemm_i8_adapters_query",
                     "igemm_i8_grouped", "igemm_i8_grouped_query", "igemm_route",
                     "igemm_route_query"]
    lib = ctypes.CDLL(ig.library_path())
    for name in names:
        assert hasattr(lib, name) and hasattr(ig, name), name


def route_desc(tokens=4, experts=8, top_k=2, groups=1, top_groups=1, group_best=1, score=0,
               renormalise=1, scale=1.0, type=0):
    return ig.RouteDesc(tokens, experts, top_k, groups, top_groups, group_best, score,
                        renormalise, scale, type)


def call_route(d, logits=P, ld=None, bias=None, ids=Q, weights=R, offsets=S, order=S, ws=None,
               ws_bytes=0):
    return ig.igemm_route(d, logits, d.experts if ld is None else ld, bias, ids, weights,
                          offsets, order, ws, ws_bytes, 0)


@pytest.mark.parametrize("bad, status", [
    (dict(tokens=-1), E), (dict(experts=0), E), (dict(top_k=0), E), (dict(top_k=9), E),
    (dict(groups=0), E), (dict(groups=3), E), (dict(groups=16), E), (dict(top_groups=0), E),
    (dict(groups=2, top_groups=3), E), (dict(group_best=0), E), (dict(group_best=3), E),
    (dict(score=2), E), (dict(renormalise=2), E), (dict(scale=float("nan")), E),
    (dict(scale=float("inf")), E), (dict(type=3), E), (dict(experts=1025), N),
    (dict(experts=128, top_k=65), N), (dict(experts=130, groups=65), N),
    (dict(tokens=1 << 31), N)])
def test_route_refuses_bad_descriptors(bad, status):
    d = route_desc(**bad)
    assert call_route(d) == status
    with pytest.raises(ig.IgemmError) as e:
        ig.igemm_route_query(d)
    assert e.value.status == status


def test_route_refuses_bad_arguments():
    d = route_desc()
    assert call_route(d, logits=0) == E
    assert call_route(d, ids=0) == E
    assert call_route(d, weights=0) == E
    assert call_route(d, ld=7) == E
    assert call_route(d, offsets=0) == E          # one of the plan's two alone
    assert call_route(d, order=0) == E
    assert call_route(d, logits=P + 2) == E       # a float at a 2-byte address
    assert call_route(route_desc(type=1), logits=P + 1) == E
    assert call_route(d, bias=P + 2) == E
    assert call_route(d, ids=Q + 2) == E
    assert call_route(d, ws=P + 16, ws_bytes=1 << 20) == E
    assert call_route(d, ws=P, ws_bytes=-1) == E
    assert call_route(d, ld=1 << 62) == N


def test_route_without_tokens_or_plan_does_nothing():
    assert call_route(route_desc(tokens=0), logits=0, ids=0, weights=0, offsets=0,
                      order=0) == ig.IGEMM_OK


def grouped_desc(rows=4, n=8, k=16, groups=3, a_rows=4, out_rows=4, slots=0, scatter=0, type=1):
    return ig.GroupedDesc(rows, n, k, groups, a_rows, out_rows, slots, scatter, type)


def call_grouped(d, offsets=S, order=None, A=P, lda=None, sa=None, B=Q, ldb=None, stride_b=None,
                 sb=None, out=R, ldo=None, ws=None, ws_bytes=0):
    return ig.igemm_i8_grouped(d, offsets, order, A, d.k if lda is None else lda, sa, B,
                               d.n if ldb is None else ldb,
                               d.k * d.n if stride_b is None else stride_b, sb, out,
                               d.n if ldo is None else ldo, ws, ws_bytes, 0)


@pytest.mark.parametrize("bad, status", [
    (dict(rows=-1), E), (dict(n=-1), E), (dict(k=-1), E), (dict(groups=-1), E),
    (dict(a_rows=-1), E), (dict(out_rows=-1), E), (dict(slots=-1), E), (dict(scatter=2), E),
    (dict(type=3), E), (dict(k=131072), N), (dict(rows=1 << 31), N), (dict(n=1 << 31), N),
    (dict(groups=65537), N)])
def test_grouped_refuses_bad_descriptors(bad, status):
    d = grouped_desc(**bad)
    assert call_grouped(d) == status
    with pytest.raises(ig.IgemmError) as e:
        ig.igemm_i8_grouped_query(d)
    assert e.value.status == status


def test_grouped_refuses_bad_arguments():
    d = grouped_desc()
    for bad in (dict(offsets=0), dict(offsets=S + 2), dict(order=S + 1), dict(A=0), dict(B=0),
                dict(out=0), dict(lda=15), dict(ldb=7), dict(ldo=7), dict(stride_b=-1),
                dict(out=R + 1), dict(sa=P + 2), dict(sb=P + 2), dict(ws=P + 16, ws_bytes=64),
                dict(ws=P, ws_bytes=-1)):
        assert call_grouped(d, **bad) == E, bad
    assert call_grouped(d, lda=1 << 30) == N          # A over 2 GiB
    assert call_grouped(d, ldb=1 << 28) == N
    assert call_grouped(d, ldo=1 << 31) == N
    assert call_grouped(d, ldo=1 << 23) == N          # 256 rows of out over 2 GiB
    assert call_grouped(d, stride_b=1 << 62) == N


def test_grouped_with_nothing_to_do():
    for none in (dict(rows=0), dict(n=0), dict(groups=0), dict(a_rows=0), dict(out_rows=0)):
        d = grouped_desc(**none)
        assert call_grouped(d, offsets=0, A=0, B=0, out=0) == ig.IGEMM_OK
        assert ig.igemm_i8_grouped_query(d) == 0


def test_combine_refusals():
    def call(tokens=4, top_k=2, n=8, type=1, Z=P, ldz=8, w=Q, ids=None, base=None, ldb=0, out=R,
             ldo=8):
        return ig.igemm_combine(tokens, top_k, n, type, Z, ldz, w, ids, base, ldb, out, ldo, 0)
    for bad in (dict(tokens=-1), dict(top_k=0), dict(n=-1), dict(type=3), dict(Z=0), dict(w=0),
                dict(out=0), dict(ldz=7), dict(ldo=7), dict(base=S, ldb=7), dict(Z=P + 1),
                dict(out=R + 1), dict(base=S + 1, ldb=8), dict(w=Q + 2), dict(ids=S + 2)):
        assert call(**bad) == E, bad
    for big in (dict(tokens=1 << 31), dict(top_k=1 << 31), dict(n=1 << 31, ldz=1 << 31,
                                                                ldo=1 << 31), dict(ldz=1 << 61)):
        assert call(**big) == N, big
    assert call(tokens=0, Z=0, w=0, out=0) == ig.IGEMM_OK
    assert call(n=0, Z=0, w=0, out=0) == ig.IGEMM_OK


def adapters_desc(m=4, n=8, k=16, adapters=2, rank=4, type=1, weight_type=1):
    return ig.AdaptersDesc(m, n, k, adapters, rank, type, weight_type)


def call_adapters(d, A=P, lda=None, sa=None, B=Q, ldb=None, sb=None, ids=S, down=P, ld_down=None,
                  up=Q, ld_up=None, sd=0, su=0, ranks=None, scaling=None, out=R, ldo=None,
                  ws=None, ws_bytes=0):
    return ig.igemm_i8_adapters(
        d, A, d.k if lda is None else lda, sa, B, d.n if ldb is None else ldb, sb, ids, down,
        d.k if ld_down is None else ld_down, sd, up, d.rank if ld_up is None else ld_up, su,
        ranks, scaling, out, d.n if ldo is None else ldo, ws, ws_bytes, 0)


@pytest.mark.parametrize("bad, status", [
    (dict(m=-1), E), (dict(n=-1), E), (dict(k=-1), E), (dict(adapters=-1), E), (dict(rank=-1), E),
    (dict(type=3), E), (dict(weight_type=0), E), (dict(weight_type=3), E), (dict(k=131072), N),
    (dict(m=1 << 31), N), (dict(rank=1025), N), (dict(adapters=1 << 31), N)])
def test_adapters_refuse_bad_descriptors(bad, status):
    d = adapters_desc(**bad)
    assert call_adapters(d) == status
    with pytest.raises(ig.IgemmError) as e:
        ig.igemm_i8_adapters_query(d)
    assert e.value.status == status


def test_adapters_refuse_bad_arguments():
    d = adapters_desc()
    for bad in (dict(A=0), dict(B=0), dict(out=0), dict(ids=0), dict(down=0), dict(up=0),
                dict(lda=15), dict(ldb=7), dict(ldo=7), dict(ld_down=15), dict(ld_up=3),
                dict(sd=-1), dict(su=-1), dict(ids=S + 2), dict(down=P + 1), dict(up=Q + 1),
                dict(ranks=S + 1), dict(scaling=S + 1), dict(sa=S + 2), dict(sb=S + 2),
                dict(out=R + 1), dict(ws=P + 16, ws_bytes=1 << 20), dict(ws=P, ws_bytes=-1)):
        assert call_adapters(d, **bad) == E, bad
    assert call_adapters(d, ld_down=1 << 30) == N
    assert call_adapters(d, ld_up=1 << 28) == N
    assert call_adapters(d, sd=1 << 62) == N
    need = ig.igemm_i8_adapters_query(d)
    assert need > 0
    assert call_adapters(d) == ig.IGEMM_ENOMEM
    assert call_adapters(d, ws=P, ws_bytes=0) == ig.IGEMM_ENOMEM
    for none in (dict(m=0), dict(n=0)):
        e = adapters_desc(**none)
        assert call_adapters(e, A=0, B=0, out=0, ids=0, down=0, up=0) == ig.IGEMM_OK
        assert ig.igemm_i8_adapters_query(e) == 0


def test_null_descriptors():
    lib = ctypes.CDLL(ig.library_path())
    q = ctypes.c_int64(7)
    assert lib.igemm_route_query(None, ctypes.byref(q)) == E
    assert lib.igemm_i8_grouped_query(None, 0, ctypes.byref(q)) == E
    assert lib.igemm_i8_adapters_query(None, 0, ctypes.byref(q)) == E
    assert lib.igemm_route_query(ctypes.byref(route_desc()), None) == E
    assert lib.igemm_i8_grouped_query(ctypes.byref(grouped_desc()), -1, ctypes.byref(q)) == E


def test_tensor_calls_check_their_tensors():
    """Wrong types, shapes and places are named before anything is enqueued."""
    a, b = torch.zeros(4, 16, dtype=torch.int8), torch.zeros(16, 8, dtype=torch.int8)
    with pytest.raises(ValueError, match="CUDA"):
        ig.adapters_i8(a, b)
    with pytest.raises(TypeError):
        ig.adapters_i8(a.int(), b)
    with pytest.raises(TypeError):
        ig.route(torch.zeros(4, 8, dtype=torch.int32), 2)
    with pytest.raises(ValueError):
        ig.route(torch.zeros(8), 2)
    with pytest.raises(TypeError):
        ig.combine(torch.zeros(4, 8), torch.zeros(2, 2, dtype=torch.float64))
    with pytest.raises(ValueError):
        ig.grouped_i8(a, b, torch.zeros(2, dtype=torch.int32))


def test_grids_past_the_largest_are_refused():
    """A launch of 2^32 threads or more is not supported: named, not a failed launch."""
    big = 1 << 30
    assert ig.igemm_combine(big, 1, 4096, 1, P, 4096, Q, None, None, 0, R, 4096, 0) == N
    d = grouped_desc(rows=(1 << 31) - 1, n=1 << 20, k=1, a_rows=1, out_rows=1, slots=1 << 30)
    assert call_grouped(d, order=S, ldo=1 << 20, ws=1 << 20, ws_bytes=1 << 62) == N
    d = adapters_desc(m=1 << 29, n=1, k=1, rank=1)
    assert call_adapters(d, ws=1 << 20, ws_bytes=1 << 62) == N


def test_arguments_that_c_would_wrap_are_refused(monkeypatch):
    monkeypatch.setattr(ig, "_expect", lambda name, what, t, *a, **kw: t.shape[-1])
    monkeypatch.setattr(ig, "_load_native", lambda: type("N", (), {"route": lambda *a: None}))
    for bad in (dict(top_k=2 ** 32 + 1), dict(groups=2 ** 32 + 1), dict(top_groups=-2 ** 32),
                dict(group_best=2 ** 31)):
        with pytest.raises(ValueError, match="does not fit"):
            ig.route(torch.zeros(4, 8), **(dict(top_k=2) | bad))


def test_reference_of_the_gpu_tests_on_hand_cases():
    ids, w, off, order = ref.route(torch.tensor([[0.0, 0.0, -float("inf"), 0.0]]), 3)
    assert ids.tolist() == [[0, 1, 3]] and np.allclose(w, 1 / 3)
    assert off.tolist() == [0, 1, 2, 2, 3] and order.tolist() == [0, 1, 2]
    # the plan of two tokens: slots by expert, ascending, then -1
    x = torch.tensor([[3.0, 1.0], [-float("inf"), 2.0]])
    ids, w, off, order = ref.route(x, 2, score="sigmoid", renormalise=False)
    assert ids.tolist() == [[0, 1], [1, -1]] and w[1, 1] == 0
    assert off.tolist() == [0, 1, 3] and order.tolist() == [0, 1, 2, -1]
    # the bias chooses, the score weighs; a group's key is its best two's sum
    x = torch.zeros(1, 4)
    ids, w, _, _ = ref.route(x, 1, bias=torch.tensor([0.0, 0.5, 0.4, 0.4]), groups=2,
                             top_groups=1, group_best=2, renormalise=False)
    assert ids.tolist() == [[2]] and w[0, 0] == 0.25
    out, wrote = ref.grouped(np.array([[1, 2]], np.int8), np.array([[[1], [1]], [[2], [3]]], np.int8),
                             [0, 0, 1], None, None, np.array([[9.0], [0.5]]), 0, False, 1,
                             np.zeros((1, 1)))
    assert out.tolist() == [[4.0]] and wrote.tolist() == [True]


def test_route_allocates_floats_whatever_the_default_type(monkeypatch):
    """The weights that the call fills are float32 also where torch's default type is
    narrower or wider (here without a device: the library's call is replaced)."""
    seen = []

    @contextlib.contextmanager
    def on(device, stream):
        yield 0
    monkeypatch.setattr(ig, "_on", on)
    monkeypatch.setattr(ig, "_expect", lambda name, what, t, *a, **kw: t.shape[-1])
    monkeypatch.setattr(ig, "igemm_route", lambda *a: seen.append(a) or ig.IGEMM_OK)
    before = torch.get_default_dtype()
    for default in (torch.bfloat16, torch.float16, torch.float64):
        try:
            torch.set_default_dtype(default)
            ids, weights, offsets, order = ig.route(torch.zeros(4, 8, dtype=torch.float32), 2,
                                                    stream=0)
        finally:
            torch.set_default_dtype(before)
        assert weights.dtype == torch.float32
        assert ids.dtype == offsets.dtype == order.dtype == torch.int32
    assert len(seen) == 3


def test_workspaces_elsewhere_are_refused():
    """A workspace in host memory, on another device or with gaps is named, not handed to
    the kernels."""
    cpu, gpu = torch.device("cpu"), torch.device("cuda", 0)
    host = torch.zeros(512, dtype=torch.uint8)
    for ws, device in ((host, gpu), (host.to("meta"), gpu), (host[::2], cpu),
                       (host[:1].expand(512), cpu), (0x10000, gpu)):
        with pytest.raises(ValueError, match="route: workspace"):
            ig._space("route", ws, 256, device)
    assert ig._space("route", host, 256, cpu) == (host, 512)
    assert ig._space("route", None, 0, gpu) == (None, 0)


def test_version_counts_these_calls():
    """A program can tell from the version that the library has them."""
    text = open(os.path.join(ROOT, "include", "igemm_rows.h")).read()
    assert "igemm_version 500" in text
    assert ig.igemm_version() >= 500
