"""Routing from logits, its gradient, quantising to 8-bit blocks and the experts' 8-bit products against their plain forms in
64 bits (oracle/operators.py).  H below is half a step of float32 at 1, 2^-24; tolerances count roundings."""
import numpy as np
import pytest
import torch

from oracle import operators as O

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11, "e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3}   # of the value
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}                                      # half the least step


@pytest.fixture(scope="module")
def B():
    from paper_2308_12066_amd import binding
    return binding


def dev(a, kind="f32"):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(TORCH[kind])


def f64(t):
    return t.detach().cpu().to(torch.float32 if t.dtype in (torch.float8_e4m3fn, torch.float8_e5m2) else t.dtype).double().numpy()


def say(*a):
    print(*a, flush=True)


# ------------------------------------------------------------------------------------ routing
def spread(z):
    """Largest distance of an available logit from its token's largest: exp's argument is rounded to half a step of it."""
    live = np.where(np.isfinite(z), z, np.nan)
    with np.errstate(all="ignore"):
        d = np.nanmax(live, 1) - np.nanmin(live, 1)
    return float(np.nan_to_num(d).max()) if z.size else 0.0


def run_route(B, z, kind, k, dtype="f32", bias=None, every=True, stream=None, **kw):
    T, E = z.shape
    r = B.Router(E, k, score=B.SCORE_SIGMOID if kind == "sigmoid" else B.SCORE_SOFTMAX, n_groups=kw.get("n_groups", 1),
                 topk_groups=kw.get("topk_groups", 0), renormalize=kw.get("renormalize", False), scale=kw.get("scale", 1.0))
    zt = z if isinstance(z, torch.Tensor) else dev(z, dtype)
    idx = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), 7.0, device="cuda")
    s = torch.full((T, E), 7.0, device="cuda") if every else None
    r.route(zt, None if bias is None else dev(bias), idx, w, s, stream)
    torch.cuda.synchronize()
    return idx.cpu().numpy(), f64(w), None if s is None else f64(s)


def check_route(B, z, kind, k, dtype="f32", bias=None, every=True, **kw):
    z = f64(dev(z, dtype))
    got = run_route(B, z, kind, k, dtype, bias, every, **kw)
    okw = dict(kw)
    okw.setdefault("topk_groups", okw.get("n_groups", 1))
    want = O.route(z, kind, k, None if bias is None else np.float32(bias).astype(np.float64), **okw)
    assert np.array_equal(got[0], want[0]), np.argwhere(got[0] != want[0])[:5]
    # exp: one rounding of its argument (spread), one step of its result; sums of up to 16 + 4 terms one after the other; three
    # more products and quotients, once for the score and once for the renormalised weight
    tol = (spread(z) + 64) * H
    assert np.all(np.abs(got[1] - want[1]) <= tol * np.abs(want[1]) + 2.0 ** -140)
    if every:
        assert np.all(np.abs(got[2] - want[2]) <= tol * want[2] + 2.0 ** -140)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k,dtype", [
    (1, 1, 1, "f32"), (1, 128, 2, "f32"), (3, 8, 8, "bf16"), (17, 7, 3, "f16"), (33, 16, 1, "f32"), (15, 17, 5, "f32"), (64, 60, 6, "bf16"),
    (5, 100, 100, "f32"), (257, 129, 17, "f32"), (40, 255, 8, "bf16"), (16, 256, 256, "f32"), (1000, 256, 8, "bf16"),
])
def test_route(B, kind, T, E, k, dtype):
    say("route", kind, T, E, k, dtype)
    g = np.random.default_rng(T * E + k)
    z = 1.5 * g.standard_normal((T, E))
    for renormalize in (False, True):
        check_route(B, z, kind, k, dtype, renormalize=renormalize, scale=2.5)
        check_route(B, z, kind, k, dtype, bias=g.integers(-30, 31, E) * 0.01, every=renormalize, renormalize=renormalize)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k,groups,keep,dtype", [
    (1, 8, 1, 8, 3, "f32"), (50, 8, 4, 2, 1, "bf16"), (33, 60, 6, 5, 3, "f32"), (20, 20, 8, 4, 2, "bf16"), (300, 256, 8, 8, 4, "bf16"),
    (300, 256, 8, 16, 2, "f16"), (7, 255, 40, 15, 5, "f32"), (100, 64, 4, 4, 4, "f32"), (9, 15, 10, 3, 2, "f32"),
])
def test_route_in_groups(B, kind, T, E, k, groups, keep, dtype):
    say("route groups", kind, T, E, k, groups, keep, dtype)
    g = np.random.default_rng(T + E + k)
    z = 1.5 * g.standard_normal((T, E))
    for bias in (None, g.standard_normal(E) * 0.05):
        check_route(B, z, kind, k, dtype, bias=bias, n_groups=groups, topk_groups=keep, renormalize=True)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,keep", [(1, 1), (4, 2)])
def test_route_with_unavailable_experts(B, kind, groups, keep):
    """Masked logits (-inf, NaN, the type's lowest value), tokens with nothing left, excluding biases, infinite logits."""
    say("route masked", kind, groups, keep)
    g = np.random.default_rng(5)
    z = g.standard_normal((40, 24)).astype(np.float32)
    z[g.random(z.shape) < 0.5] = -np.inf
    z[g.random(z.shape) < 0.1] = np.nan
    z[3] = -np.inf
    z[4] = np.nan
    z[5] = np.finfo(np.float32).min
    z[6, :] = -np.inf
    z[6, 17] = np.finfo(np.float32).min
    z[7, 20] = np.inf
    z[8, [2, 9]] = np.inf
    z[9] = -300.0 + z[9]
    z[10, ::2] = -np.inf
    z[11, 1::2] = np.nan
    bias = g.standard_normal(24).astype(np.float32) * 0.1
    out = bias.copy()
    out[[1, 7]] = -np.inf
    out[12] = np.nan
    for b in (None, bias, out):
        for renormalize in (False, True):
            check_route(B, z, kind, 6, bias=b, n_groups=groups, topk_groups=keep, renormalize=renormalize)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_route_tells_apart_what_32_bits_do_not(B, kind):
    """Selection values closer than a step of float32, and equal ones: as in 64 bits, equal ones to the lowest index."""
    say("route close", kind)
    g = np.random.default_rng(6)
    T, E = 200, 64
    z = (0.5 * g.standard_normal((T, E))).astype(np.float32)
    s = O.scores(z, kind)
    # a bias that lifts every expert's mean score to the same level leaves differences of every size; then copies of logits
    bias = (0.9 - s.mean(0)).astype(np.float32)
    z[:, 1::2] = z[:, ::2]
    z[:100, 1::2] = np.nextafter(z[:100, ::2], np.float32(9))
    bias[1::2] = bias[::2]
    for b in (bias, np.zeros(E, np.float32), np.full(E, 100.0, np.float32)):
        check_route(B, z, kind, 9, bias=b)
        check_route(B, z, kind, 4, bias=b, n_groups=16, topk_groups=3)
    check_route(B, z, kind, 9)
    check_route(B, z, kind, 4, n_groups=16, topk_groups=3)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_route_where_bias_and_score_cancel(B, kind):
    """Selection values near 0 that are sums of a score and a bias which are not: the rounding of the score decides in 32 bits."""
    say("route cancelling", kind)
    z, bias = np.array([[0.44873318, -0.00598402]], np.float32), np.array([-0.6103381, -0.4985041], np.float32)
    check_route(B, z, "sigmoid", 1, bias=bias)
    g = np.random.default_rng(11)
    T, E = 400, 64
    z = (0.7 * g.standard_normal(E) + g.standard_normal((T, E)) * 10.0 ** g.uniform(-7.5, -3, (T, 1))).astype(np.float32)
    bias = (-O.scores(z, kind).mean(0)).astype(np.float32)
    check_route(B, z, kind, 1, bias=bias)
    check_route(B, z, kind, 9, bias=bias)
    check_route(B, z, kind, 4, bias=bias, n_groups=16, topk_groups=3)
    # one candidate's value is exact, the other's carries the error of a large score
    z = np.stack([np.full(T, -40.0), 0.4 + g.standard_normal(T) * 10.0 ** g.uniform(-7.5, -5, T)], 1).astype(np.float32)
    bias = np.array([0.0, -O.scores(z, kind)[:, 1].mean()], np.float32)
    check_route(B, z, kind, 1, bias=bias)
    # groups of two whose values are a third and minus a third: their sums are near 0, they are not
    z = (0.7 * g.standard_normal(32) + g.standard_normal((T, 32)) * 10.0 ** g.uniform(-7.5, -3, (T, 1))).astype(np.float32)
    bias = (np.tile([0.34, -0.34], 16) - O.scores(z, kind).mean(0)).astype(np.float32)
    for keep in (1, 7):
        check_route(B, z, kind, 2, bias=bias, n_groups=16, topk_groups=keep)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
def test_route_takes_all_of_the_kept_groups_and_no_other(B, kind, biased):
    """All experts of the kept groups are asked for, two of them as good as equal, and the best expert of all is of another group."""
    say("route kept groups", kind, biased)
    z = np.full((8, 16), -4.0, np.float32)
    z[:, 0] = 3.0
    for t in range(8):
        z[t, 4 + t // 4 * 8:8 + t // 4 * 8] = 2.0, -1.0, -1.5, 2.0
        z[t, 4 + t // 4 * 8 + t % 4] += np.float32(2.0 ** -21)       # close to another one, or to nothing
    bias = np.full(16, 0.25, np.float32) if biased else None
    check_route(B, z, kind, 4, bias=bias, n_groups=4, topk_groups=1)
    check_route(B, z, kind, 3, bias=bias, n_groups=4, topk_groups=1)


# sigmoid(z) = 1 / (1 + exp(-z)) where exp passes what float32 holds, or 2^-126, but not yet in any way one would take: between about 88 and 139.
FAR = (-138.5, -130.0, -120.0, -112.0, -110.0, -99.0, -95.0, -92.5, -90.25, -89.0, 89.0, 90.25, 92.5, 95.0, 99.0, 110.0, 112.0, 120.0, 130.0, 138.5)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("groups,keep", [(1, 1), (4, 2)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_route_with_logits_far_from_zero(B, kind, renormalize, groups, keep, dtype):
    say("route far", kind, renormalize, groups, keep, dtype)
    g = np.random.default_rng(12)
    T, E, k = 60, 24, 6
    z = np.where(g.random((T, E)) < 0.6, g.choice(FAR, (T, E)), 1.5 * g.standard_normal((T, E)))
    z[:len(FAR)] = np.array(FAR)[:, None]                    # tokens of nothing else
    z = f64(dev(z, dtype))
    for bias in (None, (0.1 * g.standard_normal(E)).astype(np.float32)):
        got = run_route(B, z, kind, k, dtype, bias, True, n_groups=groups, topk_groups=keep, renormalize=renormalize)
        want = O.route(z, kind, k, None if bias is None else bias.astype(np.float64), groups, keep, renormalize)
        assert np.array_equal(got[0], want[0]), np.argwhere(got[0] != want[0])[:5]
        tol = (spread(z) + 64) * H                           # as in check_route; scores below the least normal number may be 0
        assert np.all(np.abs(got[1] - want[1]) <= tol * np.abs(want[1]) + 2.0 ** -126)
        assert np.all(np.abs(got[2] - want[2]) <= tol * want[2] + 2.0 ** -126)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("every", [False, True])
@pytest.mark.parametrize("renormalize", [False, True])
def test_route_backward_with_logits_far_from_zero(B, kind, every, renormalize):
    say("route backward far", kind, every, renormalize)
    g = np.random.default_rng(13)
    T, E, k = 60, 24, 6
    z = np.where(g.random((T, E)) < 0.6, g.choice(FAR, (T, E)), 1.5 * g.standard_normal((T, E)))
    z[:len(FAR)] = np.array(FAR)[:, None]
    z = f64(dev(z))
    idx = np.stack([g.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    dw, ds = g.standard_normal((T, k)).astype(np.float32), g.standard_normal((T, E)).astype(np.float32) if every else None
    r = B.Router(E, k, score=B.SCORE_SIGMOID if kind == "sigmoid" else B.SCORE_SOFTMAX, renormalize=renormalize)
    d = torch.full((T, E), 7.0, device="cuda")
    r.route_backward(dev(z), torch.from_numpy(idx).cuda(), dev(dw), None if ds is None else dev(ds), d)
    torch.cuda.synchronize()
    want, mag = O.route_loss_gradient(z, idx, kind, dw.astype(np.float64), ds, renormalize, 1.0)
    # as in check_backward; of a score or of 1 - score below 2^-126, times gradients below 2^4, all may be missing
    assert np.all(np.abs(f64(d) - want) <= 2 * (spread(z) + 64) * H * mag + H * np.abs(want) * (1 + 1e-3) + 2.0 ** -122)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("T,E,k", [(1, 8, 2), (50, 60, 6), (70, 129, 20), (100, 256, 8), (9, 256, 256)])
def test_route_writes_scores_in_place_of_the_logits(B, kind, renormalize, T, E, k):
    say("route in place", kind, renormalize, T, E, k)
    g = np.random.default_rng(T + E)
    z = 1.5 * g.standard_normal((T, E))
    for bias in (None, g.standard_normal(E) * 0.05):
        want = run_route(B, z, kind, k, bias=bias, renormalize=renormalize)
        r = B.Router(E, k, score=B.SCORE_SIGMOID if kind == "sigmoid" else B.SCORE_SOFTMAX, renormalize=renormalize)
        zt, idx, w = dev(z), torch.full((T, k), -7, dtype=torch.int32, device="cuda"), torch.full((T, k), 7.0, device="cuda")
        r.route(zt, None if bias is None else dev(bias), idx, w, zt)
        torch.cuda.synchronize()
        assert np.array_equal(idx.cpu().numpy(), want[0]) and np.array_equal(f64(w), want[1]) and np.array_equal(f64(zt), want[2])


def test_route_reads_strided_logits_on_another_stream(B):
    say("route strided")
    g = np.random.default_rng(7)
    wide = dev(g.standard_normal((70, 101)), "bf16")
    z = wide[:, 3:40]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = run_route(B, z, "softmax", 5, every=True, stream=stream)
    want = O.route(f64(z), "softmax", 5)
    assert np.array_equal(got[0], want[0])
    assert np.allclose(got[1], want[1], rtol=80 * H, atol=0) and np.allclose(got[2], want[2], rtol=80 * H, atol=0)


def test_route_on_another_stream_behind_what_filled_its_outputs(B):
    """As above, the stream waiting until the outputs have been filled; and on torch's current stream without naming it."""
    say("route stream")
    wide = dev(np.random.default_rng(7).standard_normal((70, 101)), "bf16")
    z, r, stream = wide[:, 3:40], B.Router(37, 5), torch.cuda.Stream()
    want = O.route(f64(z), "softmax", 5)
    for named in (True, False):
        idx, w, s = torch.full((70, 5), -7, dtype=torch.int32, device="cuda"), torch.full((70, 5), 7.0, device="cuda"), torch.full((70, 37), 7.0, device="cuda")
        stream.wait_stream(torch.cuda.current_stream())
        if named:
            r.route(z, None, idx, w, s, stream)
        else:
            with torch.cuda.stream(stream):
                r.route(z, None, idx, w, s)
        stream.synchronize()
        assert np.array_equal(idx.cpu().numpy(), want[0])
        assert np.allclose(f64(w), want[1], rtol=80 * H, atol=0) and np.allclose(f64(s), want[2], rtol=80 * H, atol=0)


def check_backward(B, z, kind, k, dtype, every, renormalize, scale=1.0, idx=None, strided=False):
    g = np.random.default_rng(z.size + k)
    T, E = z.shape
    z = f64(dev(z, dtype))
    if idx is None:
        idx = np.argsort(-np.nan_to_num(z, nan=-1e30, neginf=-1e30) - 0.1 * g.standard_normal(z.shape), 1)[:, :k]
    dw, ds = g.standard_normal((T, k)).astype(np.float32), (g.standard_normal((T, E)).astype(np.float32) if every else None)
    r = B.Router(E, k, score=B.SCORE_SIGMOID if kind == "sigmoid" else B.SCORE_SOFTMAX, renormalize=renormalize, scale=scale)
    out = torch.full((T, E + 3), 7.0, dtype=TORCH[dtype], device="cuda")
    d = out[:, :E] if strided else torch.full((T, E), 7.0, dtype=TORCH[dtype], device="cuda")
    r.route_backward(dev(z, dtype), torch.from_numpy(idx.astype(np.int32)).cuda(), dev(dw), None if ds is None else dev(ds), d)
    torch.cuda.synchronize()
    want, mag = O.route_loss_gradient(z, idx, kind, dw.astype(np.float64), ds, renormalize, np.float32(scale).astype(np.float64))
    # as the scores' (spread + 64), twice over: a score times a sum of terms that carry scores themselves
    tol = 2 * (spread(z) + 64) * H * mag + HALF[dtype] * np.abs(want) * (1 + 1e-3) + TINY[dtype] + 2.0 ** -130
    got = f64(d)
    assert np.all(np.abs(got - want) <= tol), (np.abs(got - want) / tol).max()
    if strided:
        assert bool((out[:, E:] == 7.0).all())


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("every", [False, True])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("T,E,k,dtype", [(1, 1, 1, "f32"), (1, 128, 2, "f32"), (19, 8, 8, "bf16"), (33, 60, 6, "f16"), (50, 129, 20, "f32"), (130, 256, 8, "bf16")])
def test_route_backward(B, kind, every, renormalize, T, E, k, dtype):
    say("route backward", kind, every, renormalize, T, E, k, dtype)
    z = 1.5 * np.random.default_rng(T + E).standard_normal((T, E))
    check_backward(B, z, kind, k, dtype, every, renormalize, 2.5, strided=E % 2 == 0)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("every", [False, True])
@pytest.mark.parametrize("renormalize", [False, True])
def test_route_backward_with_unavailable_experts(B, kind, every, renormalize):
    say("route backward masked", kind, every, renormalize)
    g = np.random.default_rng(8)
    z = g.standard_normal((12, 24)).astype(np.float32)
    z[g.random(z.shape) < 0.5] = -np.inf
    z[1] = -np.inf
    z[2] = np.nan
    z[3, 3:] = -np.inf
    z[4] = np.finfo(np.float32).min
    idx = np.stack([g.permutation(24)[:6] for _ in range(12)])
    idx[5, 2], idx[6, 0] = -1, 24                       # outside: nothing
    check_backward(B, z, kind, 6, "f32", every, renormalize, idx=idx)


def test_route_gradient_is_that_of_differences_of_the_call(B):
    """One direction a token through the forward call itself, selection held, in steps large enough for 32 bits."""
    say("route differences")
    g = np.random.default_rng(9)
    T, E, k, h = 30, 40, 4, 2.0 ** -6
    z, v, dw = (g.standard_normal(s).astype(np.float32) for s in ((T, E), (T, E), (T, k)))
    z[np.arange(T)[:, None], np.stack([g.permutation(E)[:k] for _ in range(T)])] += 4  # the selected stay selected
    for score in (B.SCORE_SOFTMAX, B.SCORE_SIGMOID):
        r = B.Router(E, k, score=score, renormalize=True)
        outs = []
        for step in (0.0, h, -h):
            idx, w = torch.zeros(T, k, dtype=torch.int32, device="cuda"), torch.zeros(T, k, device="cuda")
            r.route(dev(z + np.float32(step) * v), None, idx, w)
            outs.append((idx.cpu().numpy(), f64(w)))
        d = torch.zeros(T, E, device="cuda")
        r.route_backward(dev(z), torch.from_numpy(outs[0][0]).cuda(), dev(dw), None, d)
        got = (f64(d) * v).sum(1)
        for t in range(T):
            at = [dict(zip(o[0][t], o[1][t])) for o in outs]
            assert set(at[1]) == set(at[0]) == set(at[2])
            want = sum(dw[t, j] * (at[1][e] - at[2][e]) for j, e in enumerate(outs[0][0][t])) / (2 * h)
            # h^2 / 6 of a third derivative that is below 60 here (|v| up to 3.5, cubed, times weights), and rounding over h
            assert abs(got[t] - want) < h * h / 6 * 60 * np.abs(dw[t]).sum() + 8 * k * H / h * np.abs(dw[t]).max()


# ------------------------------------------------------------------------------------ quantising
def awkward(g, T, d):
    """Rows with blocks of zeros, tiny and huge values, values on the border between two codes, and some that are not finite."""
    x = (g.standard_normal((T, d)) * np.exp(g.standard_normal((1, d)))).astype(np.float32)
    x[0] = 0
    if T > 4:
        x[1] *= np.float32(1e-38)
        x[2] *= np.float32(2.0 ** 100)
        x[3] = 448.0 * (g.integers(-64, 65, d) / 64.0)
        x[4, d // 2] = np.inf
        x[4, d // 3] = -np.inf
        x[4, 0] = np.nan
    return x


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("T,d,dtype,copies", [
    (1, 1, "f32", 1), (1, 128, "bf16", 2), (5, 64, "f16", 1), (17, 129, "f32", 3), (33, 768, "bf16", 2), (40, 1000, "bf16", 1), (7, 1023, "f16", 8),
    (100, 2048, "f32", 1),
])
def test_quantize_rows(B, kind, T, d, dtype, copies):
    say("quantize rows", kind, T, d, dtype, copies)
    g = np.random.default_rng(T + d)
    x = awkward(g, T, d)
    if dtype == "f16":
        x = np.where(np.isfinite(x), np.clip(x, -60000, 60000), x)
    x = f64(dev(x, dtype)).astype(np.float32)
    blocks, rows = -(-d // 128), T * copies + 3
    row_of = g.permutation(rows)[:T * copies].astype(np.int32)
    if copies == 1:
        row_of = np.arange(T, dtype=np.int32)
    q = torch.full((rows, blocks * 128 + 16), 1.0, device="cuda").to(TORCH[kind])
    scale = torch.full((blocks, rows + 5), 7.0, device="cuda")
    B.quantize_rows(dev(x, dtype), q, scale[:, :rows], None if copies == 1 else torch.from_numpy(row_of).cuda(), copies)
    torch.cuda.synchronize()
    want_q, want_s = O.quantize_rows(x, kind)
    got_q, got_s = f64(q), f64(scale)
    for t in range(T):
        for j in range(copies):
            r = row_of[t * copies + j]
            assert np.array_equal(got_s[:, r], want_s[:, t].astype(np.float64))
            assert np.array_equal(got_q[r, :blocks * 128], want_q[t], equal_nan=True), (t, np.argwhere(got_q[r, :blocks * 128] != want_q[t])[:4])
    untouched = np.setdiff1d(np.arange(rows), row_of)
    assert np.all(got_q[untouched] == 1.0) and np.all(got_s[:, untouched] == 7.0) and np.all(got_q[:, blocks * 128:] == 1.0) and np.all(got_s[:, rows:] == 7.0)


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_codes_keep_the_sign_of_zero(B, kind):
    """-0 / scale is -0, in blocks of ordinary, tiny and infinite values and of zeros; of rows and of weights."""
    say("quantize minus zero", kind)
    x = np.random.default_rng(1).standard_normal((5, 256)).astype(np.float32)
    x[1] *= np.float32(1e-38)
    x[2, 3] = np.inf
    x[4] = 0.0
    x[:, ::7], x[:, 1::7] = -0.0, 0.0
    x[3, ::5] = np.float32(-1e-30)                            # goes to -0 too
    q, scale = torch.full((5, 256), 1.0, device="cuda").to(TORCH[kind]), torch.zeros(2, 5, device="cuda")
    B.quantize_rows(dev(x), q, scale)
    want, _ = O.quantize_rows(x, kind)
    got = f64(q)
    zero = want == 0
    assert np.array_equal(got, want, equal_nan=True) and np.array_equal(np.signbit(got[zero]), np.signbit(x[zero]))
    if kind == "e4m3":
        w = np.concatenate([x[:4]] * 32)[None, :, :128].copy()
        w[~np.isfinite(w)] = 1
        sf, ssf = B.fp8_weight_shapes(1, 128, 128)
        q, s = torch.zeros(sf, device="cuda").to(torch.float8_e4m3fn), torch.zeros(ssf, device="cuda")
        B.quantize_weights(dev(w), q, s)
        got, (want, _) = f64(q).reshape(-1)[O.tile_positions(128, 128)], O.quantize_weights(w)
        assert np.array_equal(got, want[0]) and np.array_equal(np.signbit(got), np.signbit(w[0]))


def test_quantize_rows_skips_rows_that_are_not_there(B):
    say("quantize rows outside")
    x = dev(np.random.default_rng(1).standard_normal((4, 128)), "bf16")
    row_of = torch.tensor([2, -1, 5, 1 << 30], dtype=torch.int32, device="cuda")
    q, scale = torch.zeros(8, 128, device="cuda").to(torch.float8_e4m3fn), torch.zeros(1, 8, device="cuda")
    B.quantize_rows(x, q[:5], scale[:, :5], row_of, 1)
    torch.cuda.synchronize()
    assert (f64(scale)[0] != 0).tolist() == [False, False, True, False, False, False, False, False]
    assert (f64(q) != 0).any(1).tolist() == [False, False, True, False, False, False, False, False]


def test_quantize_rows_reads_strided_rows_and_passes_32_bits(B):
    say("quantize rows strided")
    g = np.random.default_rng(2)
    x = g.standard_normal((6, 300)).astype(np.float32)
    for lead, dtype in ((0, "f32"), (1, "bf16"), (8, "bf16"), (3, "f32")):
        wide = torch.zeros(6, 320, dtype=TORCH[dtype], device="cuda")
        wide[:, lead:lead + 300] = dev(x, dtype)
        q, scale = torch.zeros(6, 384, device="cuda").to(torch.float8_e4m3fn), torch.zeros(3, 6, device="cuda")
        B.quantize_rows(wide[:, lead:lead + 300], q, scale)
        want_q, want_s = O.quantize_rows(f64(dev(x, dtype)).astype(np.float32), "e4m3")
        assert np.array_equal(f64(q), want_q) and np.array_equal(f64(scale), want_s)
    # rows more than 2^31 bytes apart on both sides
    far_x = torch.empty(3, (1 << 30) + 64, dtype=torch.bfloat16, device="cuda")[:, :256]
    far_q = torch.empty(3, (1 << 31) + 256, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :256]
    far_x.copy_(dev(x[:3, :256], "bf16"))
    scale = torch.zeros(2, 3, device="cuda")
    B.quantize_rows(far_x, far_q, scale)
    want_q, want_s = O.quantize_rows(f64(dev(x[:3, :256], "bf16")).astype(np.float32), "e4m3")
    assert np.array_equal(f64(far_q.contiguous()), want_q) and np.array_equal(f64(scale), want_s)


def test_quantize_rows_of_more_rows_than_a_grid_has_places(B):
    say("quantize rows many")
    T = 16 * 65535 + 2345
    x = torch.randn(T, 24, device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    q, scale = torch.full((T, 128), 1.0, device="cuda").to(torch.float8_e4m3fn), torch.zeros(1, T, device="cuda")
    B.quantize_rows(x, q, scale)
    for rows in (slice(0, 40), slice(T // 2, T // 2 + 40), slice(T - 40, T)):
        want_q, want_s = O.quantize_rows(f64(x[rows]).astype(np.float32), "e4m3")
        assert np.array_equal(f64(q[rows]), want_q) and np.array_equal(f64(scale[:, rows]), want_s)
    assert bool((scale > 0).all()) and not bool(q[:, 24:].view(torch.uint8).any())


@pytest.mark.parametrize("E,n_in,n_out,dtype", [(1, 1, 1, "f32"), (2, 128, 128, "bf16"), (3, 200, 300, "f32"), (1, 129, 257, "bf16"), (2, 384, 136, "f16"), (5, 64, 520, "bf16")])
def test_quantize_weights(B, E, n_in, n_out, dtype):
    say("quantize weights", E, n_in, n_out, dtype)
    g = np.random.default_rng(n_in + n_out)
    w = (0.02 * g.standard_normal((E, n_in, n_out))).astype(np.float32)
    w[0, 0, 0] = 3.0
    w = f64(dev(w, dtype)).astype(np.float32)
    want_q, want_s = O.quantize_weights(w)
    (sf, ssf), (sb, ssb) = B.fp8_weight_shapes(E, n_in, n_out), B.fp8_weight_shapes(E, n_out, n_in)
    new = lambda s: torch.full(s, 1.0, device="cuda").to(torch.float8_e4m3fn)  # noqa: E731
    both = [new(sf), torch.zeros(ssf, device="cuda"), new(sb), torch.zeros(ssb, device="cuda")]
    B.quantize_weights(dev(w, dtype), *both)
    for q, s, positions, codes, scales in ((both[0], both[1], O.tile_positions(n_in, n_out), want_q, want_s),
                                           (both[2], both[3], O.tile_positions(n_out, n_in), want_q.transpose(0, 2, 1), want_s.transpose(0, 2, 1))):
        flat = f64(q).reshape(E, -1)
        assert np.array_equal(flat[:, positions], codes)
        rest = np.ones(flat.shape[1], bool)
        rest[positions.ravel()] = False
        assert np.all(flat[:, rest] == 0)
        assert np.array_equal(f64(s), scales.astype(np.float64))
    one = [new(sf), torch.zeros(ssf, device="cuda")]
    B.quantize_weights(dev(w, dtype), *one)
    other = [new(sb), torch.zeros(ssb, device="cuda")]
    B.quantize_weights(dev(w, dtype), None, None, *other)
    for a, b in zip(both, one + other):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_quantize_weights_keeps_what_is_not_finite(B):
    say("quantize weights not finite")
    w = np.random.default_rng(3).standard_normal((1, 128, 128)).astype(np.float32)
    w[0, 5, 7], w[0, 9, 100] = np.nan, np.inf
    sf, ssf = B.fp8_weight_shapes(1, 128, 128)
    q, s = torch.zeros(sf, device="cuda").to(torch.float8_e4m3fn), torch.zeros(ssf, device="cuda")
    B.quantize_weights(dev(w), q, s)
    want_q, want_s = O.quantize_weights(w)
    assert np.array_equal(f64(q).reshape(1, -1)[:, O.tile_positions(128, 128)], want_q, equal_nan=True) and np.isnan(want_q).sum() == 2
    assert np.array_equal(f64(s), want_s.astype(np.float64))


# ------------------------------------------------------------------------------------ products
class Product:
    """Operands of a product, on the GPU and as the values they stand for."""

    def __init__(self, B, counts, n_in, n_out, x_kind="e4m3", seed=0):
        g = np.random.default_rng(seed + n_in + n_out + sum(counts))
        self.B, self.n_in, self.n_out, self.x_kind = B, n_in, n_out, x_kind
        E, R = len(counts), int(sum(counts))
        self.R, self.E = R, E
        x = (g.standard_normal((R, n_in)) * np.exp(0.5 * g.standard_normal((R, 1)))).astype(np.float32)
        self.x_val, self.x_s = O.quantize_rows(x, x_kind) if R else (np.zeros((0, 128 * -(-n_in // 128))), np.zeros((-(-n_in // 128), 0), np.float32))
        self.w_val, self.w_s = O.quantize_weights((0.05 * g.standard_normal((E, n_in, n_out))).astype(np.float32))
        self.offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.x_q = dev(self.x_val).to(TORCH[x_kind]) if R else torch.zeros(0, 128 * -(-n_in // 128), device="cuda").to(TORCH[x_kind])
        self.x_scale = dev(self.x_s)
        shape, _ = B.fp8_weight_shapes(E, n_in, n_out)
        flat = np.zeros((E, int(np.prod(shape[1:]))), np.float32)
        flat[:, O.tile_positions(n_in, n_out)] = self.w_val
        self.w_q, self.w_scale = dev(flat.reshape(shape)).to(torch.float8_e4m3fn), dev(self.w_s)
        self.offsets = torch.from_numpy(self.offs).cuda()

    def want(self, relu):
        return O.expert_matmul(self.x_val[:, :self.n_in], self.x_s, self.w_val, self.w_s, self.offs, relu)

    # the matrix cores' sum of 128 exact products, then two products of scales and one sum a block
    def err(self, mag):
        return (128 + 4 * -(-self.n_in // 128)) * H * mag

    def run(self, y, y_scale=None, relu=False, stream=None):
        self.B.expert_matmul(self.x_q, self.x_scale, self.w_q, self.w_scale, self.offsets, self.n_in, self.n_out, y, y_scale, relu, stream)
        torch.cuda.synchronize()

    def check(self, out, relu):
        want, mag = self.want(relu)
        err = self.err(mag)
        if out in ("e4m3", "e5m2"):
            nb = -(-self.n_out // 128)
            q = torch.full((self.R, nb * 128), 1.0, device="cuda").to(TORCH[out])
            s = torch.full((nb, self.R), 7.0, device="cuda")
            self.run(q, s, relu)
            got_q, got_s = f64(q), f64(s)
            assert np.all(got_q[:, self.n_out:] == 0)
            for b in range(nb):
                cols = slice(b * 128, min(self.n_out, (b + 1) * 128))
                amax = np.abs(want[:, cols]).max(1)
                # the scale: the largest result's error, the quotient's rounding
                assert np.all(np.abs(got_s[b] - np.maximum(amax / O.LARGEST[out], 2.0 ** -126)) <= (err[:, cols].max(1) / O.LARGEST[out]) + 2 * H * got_s[b])
                back = got_q[:, cols] * got_s[b][:, None]
                least = 2.0 ** -10 if out == "e4m3" else 2.0 ** -17      # half the type's least step
                half = np.maximum(HALF[out] * np.abs(want[:, cols]), least * got_s[b][:, None])
                # half a step of the result that was rounded, which is `err` off, and the quotient's rounding
                assert np.all(np.abs(back - want[:, cols]) <= half + (1 + HALF[out]) * err[:, cols] + 2 * H * np.abs(want[:, cols]))
        else:
            y = torch.full((self.R, self.n_out), 7.0, dtype=TORCH[out], device="cuda")
            self.run(y, None, relu)
            assert np.all(np.abs(f64(y) - want) <= err + HALF[out] * (np.abs(want) + err) + TINY[out])


COUNTS = [
    [1], [0, 1, 0], [2, 0, 3], [0, 0, 0, 0], [16], [17, 0, 15, 1], [5, 40, 0, 31, 33], [64, 65, 0, 63], [130, 1, 0, 257], [300, 0, 0, 20],
    [1] * 40, [3, 0] * 30,
]


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "x".join(map(str, c[:6])))
@pytest.mark.parametrize("n_in,n_out", [(128, 128), (1, 1), (200, 300), (640, 144), (384, 517)])
def test_expert_matmul(B, counts, n_in, n_out):
    say("matmul", counts[:6], n_in, n_out)
    p = Product(B, counts, n_in, n_out, "e5m2" if sum(counts) % 2 else "e4m3")
    for out in ("f32", "bf16", "f16", "e4m3", "e5m2"):
        p.check(out, relu=out in ("f32", "e4m3", "e5m2"))
    p.check("f32", relu=False)


@pytest.mark.parametrize("counts,n_in,n_out", [([700, 300], 1024, 640), ([90] * 20, 768, 1024), ([4, 2, 0, 7] * 16, 2048, 512), ([1, 1], 4096, 1024), ([600], 512, 2048),
                                               ([0, 1000, 9], 256, 256)])
def test_expert_matmul_of_ordinary_sizes(B, counts, n_in, n_out):
    say("matmul", counts[:6], n_in, n_out)
    p = Product(B, counts, n_in, n_out)
    for out, relu in (("bf16", False), ("f32", True), ("e4m3", True)):
        p.check(out, relu)


def test_expert_matmul_of_rows_and_results_with_strides(B):
    """Operands and results inside wider buffers, at addresses that only scalar stores reach, on another stream."""
    say("matmul strides")
    p = Product(B, [20, 0, 45, 130], 200, 132)
    want, mag = p.want(False)
    wide = torch.zeros(p.R, 384 + 16, device="cuda").to(torch.float8_e4m3fn)
    wide[:, 16:16 + 256] = p.x_q
    p.x_q = wide[:, 16:16 + 256]
    scale = torch.full((2, p.R + 9), float("nan"), device="cuda")
    scale[:, 4:4 + p.R] = p.x_scale
    p.x_scale = scale[:, 4:4 + p.R]
    stream = torch.cuda.Stream()
    for lead, width in ((0, 132), (0, 136), (1, 140), (4, 140), (2, 141)):
        for out in ("f32", "bf16"):
            y = torch.full((p.R, width), 7.0, dtype=TORCH[out], device="cuda")
            stream.wait_stream(torch.cuda.current_stream())
            p.run(y[:, lead:lead + 132], stream=stream)
            got = f64(y)
            assert np.all(np.abs(got[:, lead:lead + 132] - want) <= p.err(mag) + HALF[out] * (np.abs(want) + p.err(mag)) + TINY[out])
            assert np.all(got[:, :lead] == 7.0) and np.all(got[:, lead + 132:] == 7.0)


def test_expert_matmul_leaves_rows_of_no_expert_alone(B):
    """Offsets that end before the last row, and offsets that are no offsets: nothing outside the rows is read or written."""
    say("matmul offsets")
    p = Product(B, [20, 45, 35], 256, 192)
    want, mag = p.want(False)
    for offs, live in (([0, 20, 65, 65], 65), ([0, 20, 65, 5000], 100)):
        p.offsets = torch.tensor(offs, dtype=torch.int32, device="cuda")
        y = torch.full((p.R + 40, 192), 7.0, device="cuda")
        p.run(y[:p.R])
        got = f64(y)
        assert np.all(np.abs(got[:live] - want[:live]) <= p.err(mag[:live]) + H * np.abs(want[:live]))
        assert np.all(got[live:] == 7.0)
    for offs in ([50, -3, 1 << 30, -(1 << 30)], [99, 98, 97, 3], [-(1 << 31), (1 << 31) - 1, 0, 100]):
        p.offsets = torch.tensor(offs, dtype=torch.int32, device="cuda")
        y = torch.full((p.R + 40, 192), 7.0, device="cuda")
        p.run(y[:p.R])
        assert np.all(f64(y)[p.R:] == 7.0)


def test_expert_matmul_of_weights_and_rows_that_pass_32_bits(B):
    say("matmul far")
    p = Product(B, [20, 45], 256, 4096)
    want, mag = p.want(False)
    x = torch.empty(p.R, (1 << 26) + 16, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)   # 65 rows of 64 MiB
    x[:, :256] = p.x_q
    p.x_q = x[:, :256]
    y = torch.full((p.R, 4096), 7.0, device="cuda")
    p.run(y)
    assert np.all(np.abs(f64(y) - want) <= p.err(mag) + H * np.abs(want))
    del x
    big_E, w_val = 250, p.w_val
    shape, sshape = B.fp8_weight_shapes(big_E, 2048, 9088)      # 250 experts of 18.9 MB: 4.7 GB of codes
    q = torch.zeros(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    s = torch.ones(sshape, device="cuda")
    flat = np.zeros(int(np.prod(shape[1:])), np.float32)
    pos = O.tile_positions(2048, 9088)
    flat[pos[:256, :4096]] = w_val[0]
    q[big_E - 1] = dev(flat.reshape(shape[1:])).to(torch.float8_e4m3fn)
    rows = 20
    xq = torch.zeros(rows, 2048, device="cuda").to(torch.float8_e4m3fn)
    xq[:, :256] = dev(p.x_val[:rows]).to(torch.float8_e4m3fn)
    xs = torch.zeros(16, rows, device="cuda")
    xs[:2] = dev(p.x_s[:, :rows])
    offs = torch.full((big_E + 1,), 0, dtype=torch.int32, device="cuda")
    offs[-1] = rows
    y = torch.full((rows, 9088), 7.0, device="cuda")
    B.expert_matmul(xq, xs, q, s, offs, 2048, 9088, y)
    torch.cuda.synchronize()
    one, m1 = O.expert_matmul(p.x_val[:rows, :256], p.x_s[:, :rows], w_val[:1], np.ones_like(p.w_s[:1]), [0, rows])
    got = f64(y)
    assert np.all(np.abs(got[:, :4096] - one) <= p.err(m1) + 64 * H * m1 + H * np.abs(one)) and np.all(got[:, 4096:] == 0)


@pytest.mark.parametrize("counts", [[1, 0, 6, 2], [20, 0, 37, 23], [100, 57, 128, 115]], ids=lambda c: "x".join(map(str, c)))
def test_expert_matmul_of_more_weights_than_the_cache_holds(B, counts):
    """64 experts of 2048 x 2048, 268 MB: copies of two, so that the plain form is two matrices."""
    say("matmul large", counts)
    p = Product(B, [4, 4], 2048, 2048)
    n = 64
    counts = counts * (n // 4)
    offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    R = int(offs[-1])
    x_val, x_s = O.quantize_rows(np.random.default_rng(7).standard_normal((R, 2048)).astype(np.float32), "e4m3")
    w_q, w_scale = p.w_q.view(torch.uint8).repeat(n // 2, *[1] * (p.w_q.dim() - 1)).view(torch.float8_e4m3fn), p.w_scale.repeat(n // 2, *[1] * (p.w_scale.dim() - 1))
    y = torch.full((R, 2048), 7.0, device="cuda")
    B.expert_matmul(dev(x_val).to(torch.float8_e4m3fn), dev(x_s), w_q, w_scale, torch.from_numpy(offs).cuda(), 2048, 2048, y)
    torch.cuda.synchronize()
    got = f64(y)
    for base in (0, 1):
        rows = np.concatenate([np.arange(offs[e], offs[e + 1]) for e in range(base, n, 2)]).astype(int)
        want, mag = O.expert_matmul(x_val[rows], x_s[:, rows], p.w_val[base:base + 1], p.w_s[base:base + 1], [0, len(rows)])
        assert np.all(np.abs(got[rows] - want) <= (128 + 4 * 16) * H * mag + H * np.abs(want))


def test_expert_matmul_passes_on_what_is_not_finite(B):
    """A NaN code or scale reaches exactly the results that use it, also through ReLU and back into 8 bits."""
    say("matmul not finite")
    p = Product(B, [3, 18], 300, 260)
    p.x_q.view(torch.uint8)[5, 7] = 0x7F                      # NaN
    p.x_scale[1, 9] = float("inf")
    y = torch.zeros(p.R, 260, device="cuda")
    p.run(y, relu=True)
    bad = ~np.isfinite(f64(y))
    assert bad[5].all() and bad[9].any() and not np.delete(bad, [5, 9], 0).any()
    q, s = torch.zeros(p.R, 384, device="cuda").to(torch.float8_e4m3fn), torch.zeros(3, p.R, device="cuda")
    p.run(q, s, relu=True)
    got = f64(q)
    assert np.isnan(got[5, :260]).all() and np.isfinite(f64(s)).all() and not np.isnan(np.delete(got, [5, 9], 0)).any()


@pytest.mark.parametrize("counts", [[1, 0, 3], [17, 1] * 10, [9] * 40, [130]])
@pytest.mark.parametrize("n_in,n_out", [(256, 100), (384, 700), (1000, 520), (1025, 132), (2048, 130), (3100, 65)])
def test_expert_matmul_of_few_rows_with_its_inputs_split(B, counts, n_in, n_out):
    say("matmul split", counts[:3], n_in, n_out)
    p = Product(B, counts, n_in, n_out, "e5m2" if n_in % 2 else "e4m3")
    for out in ("f32", "bf16", "e4m3"):
        p.check(out, relu=out == "bf16")


# Enough rows for the tiled kernels, of 64 rows and of up to 256: experts without rows, with one, with a few more than a whole chunk.
TILED = {64: [20, 0, 65, 3, 64, 17, 1, 40] * 6, 256: [60, 1, 0, 17, 130, 64, 257, 31] * 5}
# The second list is for tiles of 64 rows too by now, but for its widest results.  Chunks of 64 to 256 rows and what is left over of each:
TILED["256 rows"] = [700, 1, 0, 1017, 530, 64, 1157, 31, 1500, 17, 130, 257]


@pytest.mark.parametrize("n_out", [516, 517, 520, 600, 640, 644, 1100])
def test_lists_of_rows_are_for_the_kernels_they_name(B, n_out):
    for out in (B.F32, B.BF16, B.F16, B.E4M3, B.E5M2):
        name = lambda tile: B.expert_matmul_kernel_name(sum(TILED[tile]), len(TILED[tile]), 640, n_out, out)  # noqa: E731
        assert name(64) == "matmul_tiles_kernel, 64 rows" and name("256 rows") == "matmul_tiles_kernel, 256 rows"


@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("n_in,n_out", [(1024, 640), (1300, 772)])
def test_expert_matmul_in_tiles_over_many_blocks_of_inputs(B, relu, n_in, n_out):
    """Items whose sums run over more blocks than the ring has stages, all types of results, rows of both types."""
    say("matmul tiles many blocks", relu, n_in, n_out)
    counts = TILED["256 rows"]
    assert B.expert_matmul_kernel_name(sum(counts), len(counts), n_in, n_out) == "matmul_tiles_kernel, 256 rows"
    p = Product(B, counts, n_in, n_out, "e5m2" if relu else "e4m3")
    for out in ("f32", "bf16", "f16", "e4m3", "e5m2"):
        p.check(out, relu)


@pytest.mark.parametrize("tile", TILED)
@pytest.mark.parametrize("n_in,n_out", [(200, 517), (640, 640), (517, 644), (1, 1100), (129, 520)])
def test_expert_matmul_in_tiles(B, tile, n_in, n_out):
    say("matmul tiles", tile, n_in, n_out)
    p = Product(B, TILED[tile], n_in, n_out, "e5m2" if n_in % 2 else "e4m3")
    for out in ("f32", "bf16", "f16", "e4m3", "e5m2"):
        p.check(out, relu=out in ("f32", "e4m3"))


@pytest.mark.parametrize("tile", TILED)
def test_expert_matmul_in_tiles_of_rows_and_results_with_strides(B, tile):
    say("matmul tiles strides", tile)
    n_out = 516
    p = Product(B, TILED[tile], 200, n_out)
    want, mag = p.want(False)
    wide = torch.zeros(p.R, 384 + 16, device="cuda").to(torch.float8_e4m3fn)
    wide[:, 16:16 + 256] = p.x_q
    p.x_q = wide[:, 16:16 + 256]
    scale = torch.full((2, p.R + 9), float("nan"), device="cuda")
    scale[:, 4:4 + p.R] = p.x_scale
    p.x_scale = scale[:, 4:4 + p.R]
    for lead, width in ((0, 520), (1, 524), (4, 524), (2, 521)):
        for out in ("f32", "bf16"):
            y = torch.full((p.R, width), 7.0, dtype=TORCH[out], device="cuda")
            p.run(y[:, lead:lead + n_out])
            got = f64(y)
            assert np.all(np.abs(got[:, lead:lead + n_out] - want) <= p.err(mag) + HALF[out] * (np.abs(want) + p.err(mag)) + TINY[out])
            assert np.all(got[:, :lead] == 7.0) and np.all(got[:, lead + n_out:] == 7.0)


@pytest.mark.parametrize("tile", TILED)
def test_expert_matmul_in_tiles_with_offsets_that_are_none(B, tile):
    say("matmul tiles offsets", tile)
    p = Product(B, TILED[tile], 130, 600)
    want, mag = p.want(False)
    live = int(p.offs[-2]) - 5
    for offs in (np.minimum(p.offs, live), np.where(np.arange(p.E + 1) == p.E, 1 << 30, p.offs)):
        p.offsets = torch.from_numpy(offs.astype(np.int32)).cuda()
        rows = min(int(offs[-1]), p.R)
        y = torch.full((p.R + 300, 600), 7.0, device="cuda")
        p.run(y[:p.R])
        got = f64(y)
        assert np.all(np.abs(got[:rows] - want[:rows]) <= p.err(mag[:rows]) + H * np.abs(want[:rows])) and np.all(got[rows:] == 7.0)
    g = np.random.default_rng(9)
    for offs in (g.integers(-(1 << 31), 1 << 31, p.E + 1), g.integers(-50, p.R + 50, p.E + 1), p.offs[::-1].copy()):
        p.offsets = torch.from_numpy(offs.astype(np.int32)).cuda()
        y = torch.full((p.R + 300, 600), 7.0, device="cuda")
        p.run(y[:p.R])
        assert np.all(f64(y)[p.R:] == 7.0)


@pytest.mark.parametrize("tile", TILED)
@pytest.mark.parametrize("column", [100, 200, 517])
def test_expert_matmul_in_tiles_passes_on_what_is_not_finite(B, tile, column):
    """A weight that is NaN, a row with a NaN code and a row of zeros: nothing else changes, neither result nor scale."""
    say("matmul tiles not finite", tile, column)
    p = Product(B, TILED[tile], 300, 520)
    e = p.E - 4
    rows = slice(int(p.offs[e]), int(p.offs[e + 1]))
    zero, odd = int(p.offs[4]) + 3, int(p.offs[4]) + 4        # rows of another expert
    flat = p.w_q.view(torch.uint8).reshape(p.E, -1)
    at = O.tile_positions(300, 520)[:, column]

    def run(nan):
        flat[e, torch.from_numpy(at).cuda()] = 0
        p.x_q.view(torch.uint8)[[zero, odd]] = 0
        if nan:
            flat[e, int(at[17])] = 0x7F
            p.x_q.view(torch.uint8)[odd, 7] = 0x7F
        q, s, y = torch.zeros(p.R, 640, device="cuda").to(torch.float8_e4m3fn), torch.zeros(5, p.R, device="cuda"), torch.zeros(p.R, 520, device="cuda")
        p.run(q, s)
        p.run(y)
        return f64(q)[:, :520], f64(s), f64(y)

    q0, s0, y0 = run(False)
    q1, s1, y1 = run(True)
    bad = np.zeros((p.R, 520), bool)
    bad[rows, column] = True
    bad[odd] = True
    assert np.array_equal(np.isnan(y1), bad) and np.array_equal(y1[~bad], y0[~bad])
    assert np.array_equal(np.isnan(q1), bad) and np.array_equal(q1[~bad], q0[~bad]) and np.array_equal(s1, s0)
    assert np.all(q1[zero] == 0) and np.all(s1[:, [zero, odd]] == 2.0 ** -126) and (np.delete(s1, [zero, odd], 1) > 1e-6).all()


# rows for a stream of weights, for tiles of 64 rows and for tiles of up to 256
@pytest.mark.parametrize("counts", [[3, 18], TILED[64], [700, 1, 0, 1017, 530, 64, 1157, 31, 1500, 17, 130, 257]], ids=["few", "64", "256"])
@pytest.mark.parametrize("n_out", [520, 600])
def test_codes_past_the_last_output_are_zero(B, counts, n_out):
    """Also of rows with a NaN, and where a scale is infinite and 0 times it is NaN."""
    say("matmul past the last output", counts[:3], n_out)
    p = Product(B, counts, 300, n_out)
    p.x_q.view(torch.uint8)[5, 7] = 0x7F
    p.x_scale[1, 9] = float("inf")
    for kind in ("e4m3", "e5m2"):
        nb = -(-n_out // 128)
        q, s = torch.full((p.R, nb * 128), 1.0, device="cuda").to(TORCH[kind]), torch.zeros(nb, p.R, device="cuda")
        p.run(q, s)
        assert not bool(q.view(torch.uint8)[:, n_out:].any())
        got = f64(q)[:, :n_out]
        assert np.isnan(got[5]).all() and not np.isfinite(got[9]).any() and np.isfinite(np.delete(got, [5, 9], 0)).all() and np.isfinite(f64(s)).all()


def test_gradient_of_rows_through_the_transposed_weights(B):
    """d_x = d_y . W^T by the same call on the `backward` tiles: against the formula, and against differences of the product."""
    say("matmul gradient")
    g = np.random.default_rng(4)
    counts, n_in, n_out = [30, 0, 7, 64], 300, 200
    E, R = len(counts), sum(counts)
    w = (0.05 * g.standard_normal((E, n_in, n_out))).astype(np.float32)
    sf, ssf = B.fp8_weight_shapes(E, n_in, n_out)
    sb, ssb = B.fp8_weight_shapes(E, n_out, n_in)
    new = lambda a, b: (torch.zeros(a, device="cuda").to(torch.float8_e4m3fn), torch.zeros(b, device="cuda"))  # noqa: E731
    fq, fs = new(sf, ssf)
    bq, bs = new(sb, ssb)
    B.quantize_weights(dev(w), fq, fs, bq, bs)
    dy = g.standard_normal((R, n_out)).astype(np.float32)
    dq, dscale = torch.zeros(R, 256, device="cuda").to(torch.float8_e5m2), torch.zeros(2, R, device="cuda")
    B.quantize_rows(dev(dy), dq, dscale)
    offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    dx = torch.zeros(R, n_in, device="cuda")
    B.expert_matmul(dq, dscale, bq, bs, torch.from_numpy(offs).cuda(), n_out, n_in, dx)
    q_val, s_val = O.quantize_rows(dy, "e5m2")
    w_val, w_s = O.quantize_weights(w)
    want, mag = O.expert_matmul(q_val[:, :n_out], s_val, w_val.transpose(0, 2, 1), w_s.transpose(0, 2, 1), offs)
    tol = (128 + 8) * H * mag + H * np.abs(want)
    assert np.all(np.abs(f64(dx) - want) <= tol)
    # differences: the product is linear in x, so a step of a whole block of one row (codes 1, scale h) is exact but for rounding
    back = q_val[:, :n_out] * np.repeat(s_val.T.astype(np.float64), 128, 1)[:, :n_out]     # the d_y the call saw
    for i in (0, 131, 299):
        xq, xs = torch.zeros(R, 384, device="cuda"), torch.ones(3, R, device="cuda")
        xq[:, i] = 1.0
        y = torch.zeros(R, n_out, device="cuda")
        B.expert_matmul(xq.to(torch.float8_e4m3fn), xs, fq, fs, torch.from_numpy(offs).cuda(), n_in, n_out, y)
        got = (back * f64(y)).sum(1)
        assert np.all(np.abs(got - f64(dx)[:, i]) <= tol[:, i] + 8 * H * (np.abs(back) * np.abs(f64(y))).sum(1))


# ------------------------------------------------------------------------------------ together
def moe_in_eight_bits(B, T, d, f, E, k, seed=0):
    """Buffers of one block and the calls of its step."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    w1, w2 = (0.05 * torch.randn(E, a, b, generator=g, device="cuda") for a, b in ((d, f), (f, d)))
    logits = torch.randn(T, E, generator=g, device="cuda")
    new8 = lambda *s: torch.zeros(s, device="cuda").to(torch.float8_e4m3fn)  # noqa: E731
    p = []
    for w in (w1, w2):
        qs, ss = B.fp8_weight_shapes(E, w.shape[1], w.shape[2])
        p += [new8(*qs), torch.zeros(ss, device="cuda")]
        B.quantize_weights(w, p[-2], p[-1])
    ctx = B.Context(B.make_config(d, 64, E, k, 1, T, B.BF16))
    R = T * k
    b = dict(x=x, logits=logits, idx=torch.zeros(T, k, dtype=torch.int32, device="cuda"), wt=torch.zeros(T, k, device="cuda"),
             row_of=torch.zeros(R, dtype=torch.int32, device="cuda"), offs=torch.zeros(E + 1, dtype=torch.int32, device="cuda"),
             xq=new8(R, B.fp8_blocks(d) * 128), xs=torch.zeros(B.fp8_blocks(d), R, device="cuda"), hq=new8(R, B.fp8_blocks(f) * 128),
             hs=torch.zeros(B.fp8_blocks(f), R, device="cuda"), yp=torch.zeros(R, d, dtype=torch.bfloat16, device="cuda"),
             y=torch.zeros(T, d, dtype=torch.bfloat16, device="cuda"))
    router = B.Router(E, k, renormalize=True)

    def step(stream):
        router.route(b["logits"], None, b["idx"], b["wt"], None, stream)
        ctx.group_rows(b["idx"], T, b["row_of"], b["offs"], stream)
        B.quantize_rows(b["x"], b["xq"], b["xs"], b["row_of"], k, stream)
        B.expert_matmul(b["xq"], b["xs"], p[0], p[1], b["offs"], d, f, b["hq"], b["hs"], True, stream)
        B.expert_matmul(b["hq"], b["hs"], p[2], p[3], b["offs"], f, d, b["yp"], None, False, stream)
        ctx.combine(b["yp"], b["row_of"], b["wt"], T, b["y"], None, None, stream)
    return ctx, b, (w1, w2), step


@pytest.mark.parametrize("T,d,f,E,k", [(1, 64, 256, 8, 2), (50, 128, 640, 16, 2), (300, 256, 512, 4, 3)])
def test_block_with_8_bit_experts(B, T, d, f, E, k):
    """The calls of one block one behind the other; group_rows against pgmoe_permute; the result against unquantised experts: three
    roundings of e4m3 (half a step 2^-4 of a value each) on the way, independent over hundreds of terms."""
    say("block", T, d, f, E, k)
    ctx, b, (w1, w2), step = moe_in_eight_bits(B, T, d, f, E, k)
    torch.cuda.synchronize()
    step(None)
    torch.cuda.synchronize()
    row_of, offs, xp = torch.zeros_like(b["row_of"]), torch.zeros_like(b["offs"]), torch.zeros(T * k, d, dtype=torch.bfloat16, device="cuda")
    ctx.permute(b["x"], b["idx"], T, xp, row_of, offs)
    assert torch.equal(row_of, b["row_of"]) and torch.equal(offs, b["offs"])
    idx, wt = b["idx"].long().cpu(), b["wt"].cpu().double()
    x, w1, w2 = b["x"].cpu().double(), w1.cpu().double(), w2.cpu().double()
    want = torch.stack([sum(wt[t, j] * (torch.relu(x[t] @ w1[idx[t, j]]) @ w2[idx[t, j]]) for j in range(k)) for t in range(T)])
    err = float((b["y"].cpu().double() - want).norm() / want.norm())
    assert err < 2.0 ** -4, err
    assert ctx.device_flags() == 0
    ctx.close()


def test_block_with_8_bit_experts_replays_from_a_captured_graph(B):
    say("block captured")
    T, d, f, E, k = 40, 256, 512, 8, 2
    ctx, b, _, step = moe_in_eight_bits(B, T, d, f, E, k)
    g = torch.Generator(device="cuda").manual_seed(9)
    inputs = [(torch.randn(T, d, generator=g, device="cuda").bfloat16(), torch.randn(T, E, generator=g, device="cuda")) for _ in range(3)]
    stream = torch.cuda.Stream()
    router, dl, dw = B.Router(E, k, renormalize=True), torch.zeros(T, E, device="cuda"), torch.randn(T, k, generator=g, device="cuda")

    def whole():
        step(stream)
        router.route_backward(b["logits"], b["idx"], dw, None, dl, stream)

    eager = []
    for x, z in inputs:
        b["x"].copy_(x)
        b["logits"].copy_(z)
        torch.cuda.synchronize()
        whole()
        torch.cuda.synchronize()
        eager.append((b["y"].clone(), dl.clone()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        whole()
    for rep in range(3):
        for (x, z), (y, d_logits) in zip(inputs, eager):
            b["x"].copy_(x)
            b["logits"].copy_(z)
            for name in ("y", "yp", "idx", "wt", "row_of", "offs", "xs", "hs"):
                b[name].zero_()
            dl.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(b["y"], y) and torch.equal(dl, d_logits), rep
    del graph
    ctx.close()


@pytest.fixture(scope="module")
def example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "fp8_experts.py")
    spec = importlib.util.spec_from_file_location("fp8_experts", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("T,d,f,E,k", [(1, 256, 512, 8, 2), (200, 256, 1000, 16, 2)])
def test_example_of_a_block_with_8_bit_experts(example, T, d, f, E, k):
    """examples/fp8_experts.py as it is run: replays of the captured forward give the eager bits; the result is near that of unquantised
    experts: three roundings to e4m3 (half a step 2^-4 of a value at most, on the mean a good third of it) of terms of sums."""
    say("example", T, d, f, E, k)
    errors, us, same = example.run(T, d, f, E, k, replays=3)
    assert same and us > 0
    assert errors["y"] < 2.0 ** -4 and all(np.isfinite(v) for v in errors.values()), errors


@pytest.mark.parametrize("given", [False, True])
def test_example_on_another_stream(example, given):
    """Forward and backward, inputs written late on a stream that is not the default one: the bits of the default one."""
    say("example stream", given)
    T, d, f, E, k = 200, 256, 512, 8, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    w1, w2 = (0.05 * torch.randn(E, a, b, generator=g, device="cuda") for a, b in ((d, f), (f, d)))
    x, z, dy = torch.randn(T, d, generator=g, device="cuda").bfloat16(), torch.randn(T, E, generator=g, device="cuda"), torch.randn(T, d, generator=g, device="cuda")
    block = example.Block(w1, w2, None, k, T, renormalize=True)
    want = block.forward(x, z).clone(), *block.backward(z, dy)
    torch.cuda.synchronize()
    for b in (block.y, block.y_rows, block.weight, block.idx, block.row_of, block.offsets):
        b.zero_()
    late_x, late_z, late_dy = torch.zeros_like(x), torch.zeros_like(z), torch.zeros_like(dy)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(3):
            big = big @ big * 1e-4                           # some milliseconds
        for to, of in ((late_x, x), (late_z, z), (late_dy, dy)):
            to.copy_(of)
        if not given:
            got = block.forward(late_x, late_z).clone(), *block.backward(late_z, late_dy)
    if given:
        block.forward(late_x, late_z, stream)
        got = block.backward(late_z, late_dy, stream)
        stream.synchronize()
        got = block.y.clone(), *got
    stream.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    block.close()


@pytest.mark.parametrize("T,d,f,E,k", [(1, 256, 512, 8, 2), (60, 128, 300, 16, 3)])
def test_backward_of_the_example(example, B, T, d, f, E, k):
    """Its backward against the same chain in 64 bits, from what the forward left: codes, experts, weights, results of the experts."""
    say("example backward", T, d, f, E, k)
    g = np.random.default_rng(T)
    w1, w2 = ((0.05 * g.standard_normal(s)).astype(np.float32) for s in ((E, d, f), (E, f, d)))
    x, z, dy = dev(g.standard_normal((T, d)), "bf16"), dev(g.standard_normal((T, E))), g.standard_normal((T, d)).astype(np.float32)
    block = example.Block(dev(w1), dev(w2), None, k, T, renormalize=True)
    block.forward(x, z)
    d_x, d_logits = block.backward(z, dev(dy))
    torch.cuda.synchronize()
    idx, wt, row_of, offs = block.idx.cpu().numpy(), f64(block.weight), block.row_of.cpu().numpy(), block.offsets.cpu().numpy()
    q1, s1 = O.quantize_weights(w1)
    q2, s2 = O.quantize_weights(w2)
    turn = lambda q, s: (q.transpose(0, 2, 1), s.transpose(0, 2, 1))  # noqa: E731
    d_rows = np.zeros((T * k, d), np.float32)
    d_rows[row_of] = (np.float32(wt)[:, :, None] * dy[:, None]).reshape(T * k, d)
    qv, qs = O.quantize_rows(d_rows, "e5m2")
    d_h, _ = O.expert_matmul(qv[:, :d], qs, *turn(q2, s2), offs)
    d_h = np.where(f64(block.h_q[0])[:, :f] != 0, d_h, 0)
    qv, qs = O.quantize_rows(d_h.astype(np.float32), "e5m2")
    d_rows, _ = O.expert_matmul(qv[:, :f], qs, *turn(q1, s1), offs)
    want = d_rows[row_of].reshape(T, k, d).sum(1)
    # two roundings to bfloat16 of at most 2^-8; now and then a code of e5m2 on a border, a part in a million of them
    assert np.linalg.norm(f64(d_x) - want) < 2.0 ** -8 * np.linalg.norm(want)
    d_weight = (f64(block.y_rows)[row_of].reshape(T, k, d) * dy[:, None].astype(np.float64)).sum(2)
    mag_w = (np.abs(f64(block.y_rows))[row_of].reshape(T, k, d) * np.abs(dy)[:, None]).sum(2)
    want, mag = O.route_loss_gradient(f64(z), idx, "softmax", d_weight, None, True)
    _, mag_w = O.route_loss_gradient(f64(z), idx, "softmax", mag_w, None, True)
    # the gradient of the weights is a float32 sum of d products (counted d + 2 roundings), then the gradient's own tolerance
    assert np.all(np.abs(f64(d_logits) - want) <= (d + 2) * H * mag_w + 2 * (spread(f64(z)) + 64) * H * mag + 2.0 ** -130)
    block.close()
