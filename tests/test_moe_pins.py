"""Pins of the routing oracle, and what the routing entry points refuse (no GPU)."""
import ctypes

import numpy as np
import pytest

from oracle import moe_oracle as M
from paper_2604_00317_amd import binding as B


def test_worked_example():
    x = np.array([[1.0, 3.0, 2.0, 3.0], [-np.inf, 0.0, -np.inf, -np.inf]], dtype=np.float32)
    r = M.route(x, 2)
    assert r["index"].tolist() == [[1, 3], [1, -1]]            # a tie goes to the lower index
    assert r["weight"].tolist() == [[0.5, 0.5], [1.0, 0.0]]
    assert r["counts"].tolist() == [[0, 2, 0, 1]] and r["routed"].tolist() == [2]
    z = np.exp([1.0, 3.0, 2.0, 3.0])
    np.testing.assert_allclose(r["prob_sum"][0], z / z.sum() + [0, 1, 0, 0], rtol=1e-15)
    r = M.route(x, 2, sigmoid=True, renorm=False, scale=2.0,
                bias=np.array([9.0, 0.0, 9.0, 0.0], dtype=np.float32))
    assert r["index"].tolist() == [[2, 0], [1, -1]]            # the bias chooses, and only that
    np.testing.assert_allclose(r["weight"], [[2 / (1 + np.exp(-2)), 2 / (1 + np.exp(-1))], [1.0, 0.0]],
                               rtol=1e-15)


def test_even_routing_costs_alpha_and_uneven_more():
    E, k, T = 8, 2, 16
    counts = np.full((1, E), T * k // E)
    assert M.balance_loss(counts, [T], np.full((1, E), T / E), k, 0.25)[0] == pytest.approx(0.25, rel=1e-15)
    counts[0, 0], counts[0, 1] = T, 0
    skew = np.full((1, E), T / E)
    skew[0, 0], skew[0, 1] = 2 * T / E, 0.0
    assert M.balance_loss(counts, [T], skew, k, 0.25)[0] > 0.25
    assert M.balance_loss(counts * 0, [0], skew * 0, k, 0.25)[0] == 0.0


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("bias", [False, True])
def test_gradient_against_differences(sigmoid, renorm, bias):
    """Central differences of  sum w g + sum h loss  with the choice and the counts held."""
    rng = np.random.default_rng(5)
    T, E, k, alpha, scale = 6, 7, 3, 0.5, 1.75
    ends = [0, 2, 2, 5]
    x = rng.normal(size=(T, E)).astype(np.float32)
    x[1, 3] = -np.inf
    x[4, 1:6] = -np.inf                                        # two experts left for three slots
    b = rng.normal(size=E).astype(np.float32) if bias else None
    keep = np.array([1, 1, 1, 0, 1, 1])
    g, h = rng.normal(size=(T, k)), rng.normal(size=3)
    r = M.route(x, k, sigmoid, renorm, scale, b, keep, ends)
    dx, _ = M.route_backward(x, r["index"], r["weight"], sigmoid, renorm, scale, keep, ends,
                             g, alpha, r["counts"], r["routed"], h)

    def value(z):
        total = 0.0
        for s in range(3):
            P = np.zeros(E)
            for t in range(ends[s], ends[s + 1]):
                if not keep[t]:
                    continue
                sc = np.where(np.isneginf(z[t]), 0.0, 1 / (1 + np.exp(-z[t])) if sigmoid else np.exp(z[t]))
                P += sc / sc.sum()
                idx = [e for e in r["index"][t] if e >= 0]
                if renorm:
                    w = scale * sc[idx] / sc[idx].sum()
                else:
                    w = scale * sc[idx] / (1.0 if sigmoid else sc.sum())
                total += float((w * g[t, :len(idx)]).sum())
            if r["routed"][s]:
                total += h[s] * M.balance_loss(r["counts"][s:s + 1], r["routed"][s:s + 1], P[None], k, alpha)[0]
        return total

    assert np.isnan(dx[5]).all() and not dx[3].any()
    z, step = x.astype(np.float64), 1e-6
    for t in range(5):
        for e in range(E):
            if np.isneginf(z[t, e]):
                assert dx[t, e] == 0.0
                continue
            up, down = z.copy(), z.copy()
            up[t, e] += step
            down[t, e] -= step
            # curvature: third derivatives of order 1 times step^2; cancellation: 2^-53 / step
            assert dx[t, e] == pytest.approx((value(up) - value(down)) / (2 * step), abs=2e-9)


def test_counts_and_traffic_by_hand():
    index = np.array([[0, 1], [2, -1], [3, 3], [1, 2], [9, 0]], dtype=np.int32)
    place = np.array([0, 0, 1, 1])
    per_e, per_r = M.counts(index, 4, [0, 2, 2, 4], place, 2)
    assert per_e.tolist() == [[1, 1, 1, 0], [0, 0, 0, 0], [0, 1, 1, 2]]
    assert per_r.tolist() == [[1, 1], [0, 0], [1, 2]]
    rt = np.array([[[5, 1, 2], [3, 6, 4], [7, 8, 9]]])
    assert M.traffic(rt, 10.0).tolist() == [[10, 20, 30, 40, 70, 80]]
    assert M.traffic(rt, 10.0, way_back=True).tolist() == [[30, 70, 10, 80, 20, 40]]
    t = M.traffic(rt, 1.0, [2, 0, 3], [0, 0, 1])
    assert t[0, :2].tolist() == [7, 5] and np.isnan(t[0, 2])


# ---- refusals, before any device call --------------------------------------------------------

P = ctypes.c_void_p(4096)                 # never looked at: every call below is refused first

ROUTE = dict(tokens=4, experts=8, top_k=2, flags=0, dtype=0, logits=P, stride=8, bias=None, keep=None,
             scale=1.0, n_seg=1, seg=None, index=P, weight=P, counts=None, routed=None,
             prob=None, scratch=None, nbytes=0, stream=None)
SUMS = dict(ROUTE, counts=P, routed=P, prob=P, scratch=P, nbytes=1 << 20)


@pytest.mark.parametrize("base,change,status", [
    (ROUTE, dict(tokens=-1), 1), (ROUTE, dict(experts=0), 1), (ROUTE, dict(experts=2049, stride=4096), 4),
    (ROUTE, dict(top_k=0), 1), (ROUTE, dict(top_k=9), 1), (ROUTE, dict(top_k=17, experts=64, stride=64), 4),
    (ROUTE, dict(flags=4), 1), (ROUTE, dict(dtype=3), 1), (ROUTE, dict(dtype=-1), 1),
    (ROUTE, dict(logits=None), 1), (ROUTE, dict(index=None), 1), (ROUTE, dict(weight=None), 1),
    (ROUTE, dict(stride=7), 1), (ROUTE, dict(scale=0.0), 1), (ROUTE, dict(scale=float("nan")), 1),
    (ROUTE, dict(scale=float("inf")), 1), (ROUTE, dict(scale=1e-39), 1), (ROUTE, dict(tokens=0x7FFF0001), 4),
    (ROUTE, dict(scale=-1.0), 1), (ROUTE, dict(n_seg=0), 1),
    (ROUTE, dict(n_seg=2), 1), (ROUTE, dict(n_seg=(1 << 20) + 1, seg=P), 4),
    (ROUTE, dict(counts=P), 1), (SUMS, dict(prob=None), 1), (SUMS, dict(scratch=None), 1),
    (SUMS, dict(scratch=ctypes.c_void_p(4100)), 1), (SUMS, dict(nbytes=16), 1),
])
def test_route_refuses(base, change, status):
    lib = B.load_library()
    assert lib.nimble_moe_route(*dict(base, **change).values()) == status
    assert lib.nimble_last_error().decode()


LOSS = dict(n_seg=1, experts=8, top_k=2, counts=P, routed=P, prob=P, alpha=1.0, loss=P, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(n_seg=0), 1), (dict(experts=0), 1), (dict(top_k=0), 1), (dict(top_k=9), 1),
    (dict(experts=2049), 4), (dict(n_seg=1 << 21), 4), (dict(counts=None), 1), (dict(routed=None), 1),
    (dict(prob=None), 1), (dict(loss=None), 1), (dict(alpha=float("inf")), 1)])
def test_loss_refuses(change, status):
    assert B.load_library().nimble_moe_balance_loss(*dict(LOSS, **change).values()) == status


BACK = dict(tokens=4, experts=8, top_k=2, flags=0, dtype=0, logits=P, stride=8, keep=None, scale=1.0,
            n_seg=1, seg=None, index=P, weight=P, gw=P, alpha=1.0, counts=P, routed=P, gl=P,
            grad=P, gstride=8, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), 1), (dict(top_k=9), 1), (dict(flags=8), 1), (dict(dtype=5), 1), (dict(stride=7), 1),
    (dict(gstride=7), 1), (dict(logits=None), 1), (dict(index=None), 1), (dict(weight=None), 1),
    (dict(grad=None), 1), (dict(counts=None), 1), (dict(routed=None), 1),
    (dict(gl=None), 1), (dict(scale=1e-39), 1), (dict(tokens=0x7FFFFFFF), 4), (dict(alpha=float("nan")), 1), (dict(scale=0.0), 1), (dict(n_seg=3), 1),
    (dict(experts=4000, stride=4000, gstride=4000), 4)])
def test_backward_refuses(change, status):
    assert B.load_library().nimble_moe_route_backward(*dict(BACK, **change).values()) == status


COUNT = dict(tokens=4, top_k=2, index=P, experts=8, n_seg=1, seg=None, place=P, ranks=2, counts=P,
             rank_tokens=P, scratch=P, nbytes=1 << 20, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), 1), (dict(top_k=0), 1), (dict(top_k=17), 4), (dict(experts=0), 1),
    (dict(tokens=0x7FFF0001), 4),
    (dict(experts=2049), 4), (dict(index=None), 1), (dict(n_seg=0), 1), (dict(n_seg=2), 1),
    (dict(counts=None, rank_tokens=None), 1), (dict(place=None), 1), (dict(ranks=0), 1),
    (dict(ranks=-1), 1), (dict(ranks=4097), 4), (dict(scratch=None), 1), (dict(nbytes=8), 1)])
def test_counts_refuse(change, status):
    assert B.load_library().nimble_moe_counts(*dict(COUNT, **change).values()) == status


TRAFFIC = dict(batch=1, ranks=4, tokens=P, nbytes=2.0, n_comm=12, src=None, dst=None, flags=0, out=P,
               stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=0), 1), (dict(ranks=0), 1), (dict(ranks=5000), 4), (dict(n_comm=11), 1),
    (dict(n_comm=0), 1), (dict(src=P), 1), (dict(dst=P), 1), (dict(flags=2), 1), (dict(tokens=None), 1),
    (dict(out=None), 1), (dict(nbytes=-1.0), 1), (dict(nbytes=float("inf")), 1),
    (dict(nbytes=float("nan")), 1), (dict(batch=1 << 28), 4)])
def test_traffic_refuses(change, status):
    assert B.load_library().nimble_moe_traffic(*dict(TRAFFIC, **change).values()) == status


def test_scratch_sizes():
    assert B.nimble_moe_route_scratch_bytes(0, 8) >= 0
    assert B.nimble_moe_route_scratch_bytes(-1, 8) == -1 == B.nimble_moe_route_scratch_bytes(4, 4096)
    assert B.nimble_moe_route_scratch_bytes(4, 8, 0) == -1
    assert B.nimble_moe_counts_scratch_bytes(4, 17, 8) == -1 == B.nimble_moe_counts_scratch_bytes(4, 2, 8, -1)
    most = 0x7FFF0000
    big = B.nimble_moe_route_scratch_bytes(most, 2048, 1 << 20)
    assert big > 1 << 32 and B.nimble_moe_counts_scratch_bytes(most, 16, 2048, 4096, 1 << 20) > 1 << 32
    assert B.nimble_moe_route_scratch_bytes(most + 1, 8) == -1 == B.nimble_moe_counts_scratch_bytes(most + 1, 2, 8)


def test_binding_refuses_host_tensors():
    import torch
    x, i, w = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    with pytest.raises(TypeError):
        B.nimble_moe_route(x, i, w)
    with pytest.raises(ValueError):
        B.nimble_moe_route(x.double(), i, w)
    with pytest.raises(TypeError):
        B.nimble_moe_counts(i, 8, i)


def test_scratch_of_sizes_that_do_not_fit_32_bits():
    for at in range(3):
        sizes = [4, 8, 1]
        sizes[at] += 1 << 32
        assert B.nimble_moe_route_scratch_bytes(*sizes) == -1
    for at in range(5):
        sizes = [4, 2, 8, 4, 1]
        sizes[at] += 1 << 32
        assert B.nimble_moe_counts_scratch_bytes(*sizes) == -1


def test_without_torchs_bare_device_and_stream(monkeypatch):
    """Where torch lacks the bare functions, the public ones are asked."""
    import torch
    from types import SimpleNamespace
    B.load_library()
    for name in ("_lib", "_current_gpu", "_raw_stream"):
        monkeypatch.setattr(B, name, None)
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 5)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda gpu: SimpleNamespace(cuda_stream=1000 + gpu))
    B.load_library()
    assert B._current_gpu() == 5 and B._raw_stream(7) == 1007
