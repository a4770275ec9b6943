"""Rows there and back with weights, the way back through a ReLU kept in 8 bits, and the gradient of the experts' matrices, against
their plain forms in 64 bits (oracle/operators.py).  H is half a step of float32 at 1, 2^-24; tolerances count roundings."""
import numpy as np
import pytest
import torch

from oracle import operators as O

pytestmark = pytest.mark.gpu

H = 2.0 ** -24
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}                                         # of the value
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}                                      # half the least step
DTYPES = ("f32", "bf16", "f16")


@pytest.fixture(scope="module")
def B():
    from paper_2308_12066_amd import binding
    return binding


def dev(a, kind="f32"):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(TORCH[kind])


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def f64(t):
    return t.detach().cpu().to(torch.float32 if t.element_size() == 1 else t.dtype).double().numpy()


def say(*a):
    print(*a, flush=True)


def near(got, want, err, kind):
    """|got - want|: `err` before the last rounding, and that."""
    got = f64(got) if isinstance(got, torch.Tensor) else got
    with np.errstate(invalid="ignore"):
        assert np.all(np.abs(got - want) <= err + HALF[kind] * (np.abs(want) + err) + TINY[kind]), np.nanmax(np.abs(got - want) - err - HALF[kind] * np.abs(want))


def entries(g, T, k, dropped=0, spare=0):
    """row_of [T * k] and the rows there are: some entries name no row, some rows have no entry."""
    row_of = g.permutation(T * k + spare)[:T * k].astype(np.int32)
    if dropped:
        row_of[g.permutation(T * k)[:dropped]] = g.choice(np.array([-1, T * k + spare, -2 ** 31, 2 ** 31 - 1], np.int32), dropped)
    return row_of, T * k + spare


def check_codes(q, s, values, cols, kind, pow2, named=None):
    """Codes and scales are a function of the float32 values: equal."""
    want_q, want_s = O.quantize_rows(values.astype(np.float32), kind, pow2)
    named = np.ones(len(values), bool) if named is None else named
    got_q, got_s = f64(q), f64(s)
    assert np.array_equal(got_q[named], want_q[named], equal_nan=True) and np.array_equal(got_s[:, named], want_s[:, named].astype(np.float64))
    assert np.all(got_q[named][:, cols:] == 0)
    assert np.all(got_q[~named] == 1) and np.all(got_s[:, ~named] == 7)


def codes_for(rows, cols, kind):
    nb = -(-cols // 128)
    return torch.full((rows, nb * 128), 1.0, device="cuda").to(TORCH[kind]), torch.full((nb, rows), 7.0, device="cuda")


SHAPES = [(1, 1, 1), (1, 2, 1024), (3, 2, 130), (7, 3, 516), (40, 8, 64), (17, 1, 4100), (300, 4, 520), (5, 300, 24), (1100, 1, 96)]


# ------------------------------------------------------------------------------------ dispatch
@pytest.mark.parametrize("T,k,d", SHAPES)
@pytest.mark.parametrize("weighed", [False, True])
def test_dispatch_rows(B, T, k, d, weighed):
    say("dispatch", T, k, d, weighed)
    g = np.random.default_rng(T + d + k)
    for n, (x_kind, kind, q_kind, pow2) in enumerate((("bf16", "bf16", None, False), ("f32", "bf16", "e5m2", True), ("f16", "f32", "e4m3", False), ("bf16", None, "e4m3", True),
                                                       ("f32", "f16", "e5m2", False), ("f32", "f32", None, False))):
        row_of, R = entries(g, T, k, dropped=(T * k) // 5, spare=n % 3)
        x = dev(g.standard_normal((T, d)) * np.exp(g.standard_normal((T, 1))), x_kind)
        w = g.standard_normal((T, k)).astype(np.float32) if weighed else None
        rows = torch.full((R, d), 7.0, device="cuda").to(TORCH[kind]) if kind else None
        q, s = codes_for(R, d, q_kind) if q_kind else (None, None)
        B.dispatch_rows(x, ints(row_of), rows, q, s, None if w is None else dev(w), pow2)
        torch.cuda.synchronize()
        want = O.dispatch_rows(f64(x), row_of, R, w)
        named = ~np.isnan(want[:, 0])
        if kind:
            near(f64(rows)[named], want[named], H * np.abs(want[named]) + 2.0 ** -150, kind)
            assert np.all(f64(rows)[~named] == 7)
        if q_kind:  # the product in 64 bits, rounded to 32, is the float32 product
            check_codes(q, s, np.nan_to_num(want), d, q_kind, pow2, named)


def test_dispatch_of_values_that_are_not_finite(B):
    """They stay in their columns, and a weight that is not finite leaves the codes past the last column zero."""
    say("dispatch not finite")
    d = 200
    x = np.random.default_rng(1).standard_normal((6, d)).astype(np.float32)
    x[0, 3], x[1, 130], x[2, :], x[3, 5] = np.inf, np.nan, 0.0, -np.inf
    w = np.array([[1, 2], [1, 0], [np.inf, 1], [0, np.nan], [np.inf, 3], [1e-45, 1e38]], np.float32)
    row_of = np.arange(12, dtype=np.int32)[::-1].copy()
    rows = torch.zeros(12, d, device="cuda")
    for kind in ("e4m3", "e5m2"):
        for pow2 in (False, True):
            q, s = codes_for(12, d, kind)
            B.dispatch_rows(dev(x), ints(row_of), rows, q, s, dev(w), pow2)
            torch.cuda.synchronize()
            with np.errstate(all="ignore"):
                want = np.zeros((12, d), np.float32)
                want[row_of] = (np.float32(w)[:, :, None] * x[:, None]).reshape(12, d)
                assert np.array_equal(f64(rows), want.astype(np.float64), equal_nan=True)
                check_codes(q, s, want, d, kind, pow2)


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("d", [1, 128, 300])
def test_scales_that_are_powers_of_two(B, kind, d):
    """quantize_rows and dispatch_rows give the same codes, those of the plain form: at the borders of a scale, for zeros, tiny and huge values."""
    say("pow2", kind, d)
    g = np.random.default_rng(d)
    x = (g.standard_normal((64, d)) * np.exp2(g.integers(-140, 120, (64, 1)))).astype(np.float32)
    top = np.float32(O.LARGEST[kind])
    x[:8] = 0
    x[1:8, 0] = [top, np.nextafter(top, np.float32(1e9)), np.nextafter(top, np.float32(0)), -top * 2, 1e-45, 2.0 ** -126, 3.3e38]
    q, s = codes_for(64, d, kind)
    B.quantize_rows(dev(x), q, s, pow2=True)
    p, t = codes_for(64, d, kind)
    B.dispatch_rows(dev(x), ints(np.arange(64)), None, p, t, pow2=True)
    torch.cuda.synchronize()
    check_codes(q, s, x, d, kind, True)
    assert torch.equal(q.view(torch.uint8), p.view(torch.uint8)) and torch.equal(s, t)


def test_expert_matmul_with_scales_that_are_powers_of_two(B):
    """Quantised results of each of the product's kernels: codes times scales are the float32 results to half a step, every scale the least power for
    the largest result, give or take a rounding of that."""
    say("matmul pow2")
    g = np.random.default_rng(8)
    for counts, n_in, n_out in (([3, 0, 5], 200, 300), ([64] * 40, 200, 517), ([1500] * 40, 130, 520)):
        E, R = len(counts), sum(counts)
        names = {B.expert_matmul_kernel_name(R, E, n_in, n_out, B.E4M3)}
        w = dev(0.05 * g.standard_normal((E, n_in, n_out)))
        qs, ss = B.fp8_weight_shapes(E, n_in, n_out)
        wq, ws = torch.zeros(qs, device="cuda").to(torch.float8_e4m3fn), torch.zeros(ss, device="cuda")
        B.quantize_weights(w, wq, ws)
        xq, xs = codes_for(R, n_in, "e4m3")
        B.quantize_rows(dev(g.standard_normal((R, n_in))), xq, xs, pow2=True)
        offs = ints(np.concatenate([[0], np.cumsum(counts)]))
        y = torch.zeros(R, n_out, device="cuda")
        B.expert_matmul(xq, xs, wq, ws, offs, n_in, n_out, y, relu=True)
        for kind in ("e4m3", "e5m2"):
            q, s = codes_for(R, n_out, kind)
            B.expert_matmul(xq, xs, wq, ws, offs, n_in, n_out, q, s, relu=True, pow2=True)
            torch.cuda.synchronize()
            v, c, sc = f64(y), f64(q), f64(s)
            assert np.all(np.frexp(sc)[0] == 0.5) and np.all(c[:, n_out:] == 0), names
            half, least = (2.0 ** -4, 2.0 ** -10) if kind == "e4m3" else (2.0 ** -3, 2.0 ** -17)
            for b in range(sc.shape[0]):
                cols = slice(b * 128, min(n_out, b * 128 + 128))
                amax = np.abs(v[:, cols]).max(1)
                # the float32 results of both calls are sums in the same order or in another: each within n_in + 4 roundings of terms whose magnitudes sum to a few amax
                slack = 1 + 64 * n_in * H
                assert np.all(amax <= O.LARGEST[kind] * sc[b] * slack) and np.all((amax * slack > O.LARGEST[kind] * sc[b] / 2) | (sc[b] == 2.0 ** -126)), names
                assert np.all(np.abs(c[:, cols] * sc[b][:, None] - v[:, cols]) <= np.maximum(half * np.abs(v[:, cols]), least * sc[b][:, None]) + 64 * n_in * H * amax[:, None]), names


# ------------------------------------------------------------------------------------ combine
@pytest.mark.parametrize("T,k,d", SHAPES)
@pytest.mark.parametrize("weighed,added", [(False, False), (True, False), (True, True)])
def test_combine_rows(B, T, k, d, weighed, added):
    say("combine", T, k, d, weighed, added)
    g = np.random.default_rng(T + d + k)
    for n, (r_kind, kind) in enumerate((("bf16", "bf16"), ("f32", "f16"), ("f16", "f32"), ("bf16", "f32"))):
        row_of, R = entries(g, T, k, dropped=(T * k) // 4, spare=n % 2)
        rows = dev(g.standard_normal((R, d)), r_kind)
        w = g.standard_normal((T, k)).astype(np.float32) if weighed else None
        add = dev(g.standard_normal((T, d)), kind) if added else None
        y = torch.full((T, d), 7.0, device="cuda").to(TORCH[kind])
        B.combine_rows(rows, ints(row_of), y, None if w is None else dev(w), add)
        torch.cuda.synchronize()
        want, mag = O.combine_rows(f64(rows), row_of, T, w, None if add is None else f64(add))
        near(y, want, (k + 1) * H * mag, kind)
        if added:  # in place
            B.combine_rows(rows, ints(row_of), add, None if w is None else dev(w), add)
            torch.cuda.synchronize()
            assert torch.equal(add, y)


def test_combine_skips_dropped_copies_whatever_their_weights(B):
    say("combine dropped")
    rows = torch.full((4, 40), float("nan"), device="cuda")
    rows[1] = 2.0
    w = torch.tensor([[float("nan"), 3.0], [float("inf"), float("nan")]], device="cuda")
    y = torch.full((2, 40), 7.0, device="cuda")
    B.combine_rows(rows, ints([-1, 1, 4, 2 ** 31 - 1]), y, w)
    torch.cuda.synchronize()
    assert torch.all(y[0] == 6) and torch.all(y[1] == 0)
    empty = torch.zeros(0, 40, device="cuda")
    B.combine_rows(empty, ints([0, 1, 2, 3]), y, w, torch.ones_like(y))          # no rows at all
    torch.cuda.synchronize()
    assert torch.all(y == 1)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,d", [(1, 1, 512), (1, 2, 1024), (64, 2, 768), (1100, 8, 2048), (1500, 2, 512)])
def test_both_combines_give_the_same_bits(B, T, k, d, kind):
    """The context's and the one without, of the same rows."""
    say("both combines", T, k, d, kind)
    g = np.random.default_rng(T)
    row_of, R = entries(g, T, k)
    rows, of, w = dev(g.standard_normal((R, d)), kind), ints(row_of), dev(g.random((T, k)))
    ctx = B.Context(B.make_config(d, 64, 16, k, 1, T, B.BF16 if kind == "bf16" else B.F32))
    y, z = (torch.full((T, d), 7.0, device="cuda").to(TORCH[kind]) for _ in range(2))
    ctx.combine(rows, of, w, T, y, stream=torch.cuda.current_stream())
    B.combine_rows(rows, of, z, w)
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    ctx.close()


# ------------------------------------------------------------------------------------ combine's gradient
@pytest.mark.parametrize("T,k,d", SHAPES)
@pytest.mark.parametrize("weighed", [False, True])
def test_combine_rows_backward(B, T, k, d, weighed):
    say("combine backward", T, k, d, weighed)
    g = np.random.default_rng(T + d + k)
    for n, (x_kind, kind, q_kind, values) in enumerate((("bf16", "bf16", None, True), ("f32", "bf16", "e5m2", True), ("f16", "f32", "e4m3", False), ("f32", "f16", None, False),
                                                        ("bf16", "f32", "e5m2", True))):
        row_of, R = entries(g, T, k, dropped=(T * k) // 5, spare=n % 3)
        d_y, rows = dev(g.standard_normal((T, d)), x_kind), dev(g.standard_normal((R, d)), kind)
        w = g.standard_normal((T, k)).astype(np.float32) if weighed else None
        wt = None if w is None else dev(w)
        d_rows = torch.full((R, d), 7.0, device="cuda").to(TORCH[kind]) if values else None
        q, s = codes_for(R, d, q_kind) if q_kind else (None, None)
        d_w = torch.full((T, k), 7.0, device="cuda")
        B.combine_rows_backward(d_y, rows, ints(row_of), wt, d_rows, d_w, q, s, pow2=bool(n % 2))
        torch.cuda.synchronize()
        want = O.dispatch_rows(f64(d_y), row_of, R, w)
        named = ~np.isnan(want[:, 0])
        if values:
            near(f64(d_rows)[named], want[named], H * np.abs(want[named]) + 2.0 ** -150, kind)
            assert np.all(f64(d_rows)[~named] == 7)
        if q_kind:
            check_codes(q, s, np.nan_to_num(want), d, q_kind, bool(n % 2), named)
        want_w, mag = O.combine_weight_gradient(f64(d_y), f64(rows), row_of)
        # a lane's products one after the other, six sums over the lanes, three over the wavefronts
        near(d_w, want_w, (8 * -(-d // 512) + 9) * H * mag + 2.0 ** -140, "f32")
        if values:  # without the weights' gradient the rows are not asked for: same bits
            again = torch.full_like(d_rows, 7.0)
            B.combine_rows_backward(d_y, None, ints(row_of), wt, again)
            torch.cuda.synchronize()
            assert torch.equal(again, d_rows)


def test_gradients_of_a_combine_are_those_of_differences_of_the_call(B):
    """Combine is linear in rows and weights: a step of one value is off by roundings alone."""
    say("combine differences")
    g = np.random.default_rng(3)
    T, k, d = 6, 3, 40
    row_of, R = entries(g, T, k, dropped=3)
    rows, w, c = g.standard_normal((R, d)).astype(np.float32), g.standard_normal((T, k)).astype(np.float32), g.standard_normal((T, d)).astype(np.float32)
    d_rows, d_w = torch.zeros(R, d, device="cuda"), torch.zeros(T, k, device="cuda")
    B.combine_rows_backward(dev(c), dev(rows), ints(row_of), dev(w), d_rows, d_w)

    def loss(rows, w):
        y = torch.zeros(T, d, device="cuda")
        B.combine_rows(dev(rows), ints(row_of), y, dev(w))
        torch.cuda.synchronize()
        return (f64(y) * c).sum()
    # values of order one: k + 1 roundings of each of T * d sums of k terms, over the step of 2
    tol = (k + 1) * H * T * d * k * 8 / 2
    for r, i in ((0, 0), (7, 39), (R - 1, 11)):
        step = np.zeros_like(rows)
        step[r, i] = 1
        assert abs((loss(rows + step, w) - loss(rows - step, w)) / 2 - f64(d_rows)[r, i]) <= tol
    for t, j in ((0, 0), (3, 2), (5, 1)):
        step = np.zeros_like(w)
        step[t, j] = 1
        assert abs((loss(rows, w + step) - loss(rows, w - step)) / 2 - f64(d_w)[t, j]) <= tol


def test_rows_there_and_back_is_the_transposed_map(B):
    """<dispatch(x), g> = <x, combine(g)>, both with the same weights and dropped copies: the calls are each other's gradients."""
    say("transposed")
    g = np.random.default_rng(4)
    T, k, d = 50, 3, 72
    row_of, R = entries(g, T, k, dropped=20, spare=5)
    x, r, w = g.standard_normal((T, d)), g.standard_normal((R, d)), g.standard_normal((T, k))
    there, back = torch.zeros(R, d, device="cuda"), torch.zeros(T, d, device="cuda")
    B.dispatch_rows(dev(x), ints(row_of), there, weight=dev(w))
    B.combine_rows(dev(r), ints(row_of), back, dev(w))
    torch.cuda.synchronize()
    x, r = x.astype(np.float32).astype(np.float64), r.astype(np.float32).astype(np.float64)
    mag = (np.abs(f64(there)) * np.abs(r)).sum()
    assert abs((f64(there) * r).sum() - (x * f64(back)).sum()) <= (k + 3) * H * mag


# ------------------------------------------------------------------------------------ through the ReLU
@pytest.mark.parametrize("R,n", [(1, 1), (1, 4096), (3, 130), (17, 516), (130, 64), (40, 2050), (257, 384)])
@pytest.mark.parametrize("h_kind", ["e4m3", "e5m2"])
def test_relu_backward(B, R, n, h_kind):
    say("relu", R, n, h_kind)
    g = np.random.default_rng(R + n)
    width = -(-n // 128) * 128
    for x_kind, kind, q_kind, pow2 in (("f32", "bf16", "e5m2", True), ("bf16", "bf16", None, False), ("f16", None, "e4m3", False), ("bf16", "f32", "e5m2", False), ("f32", "f32", None, False),
                                       ("f32", "f16", "e4m3", True)):
        codes = torch.from_numpy(g.integers(0, 256, (R, width)).astype(np.uint8)).cuda().view(TORCH[h_kind])     # every code there is
        d_h = dev(g.standard_normal((R, n)), x_kind)
        blocked = (f64(codes)[:, :n] <= 0) & (g.random((R, n)) < 0.1)
        d_h[torch.from_numpy(blocked).cuda()] = float("nan") if R % 2 else float("inf")
        want = O.relu_backward(f64(d_h), f64(codes)[:, :n])
        d_pre = torch.full((R, n), 7.0, device="cuda").to(TORCH[kind]) if kind else None
        q, s = codes_for(R, n, q_kind) if q_kind else (None, None)
        B.relu_backward(d_h, codes, d_pre, q, s, pow2)
        torch.cuda.synchronize()
        if kind:
            near(d_pre, want, 0, kind)
        if q_kind:
            check_codes(q, s, want, n, q_kind, pow2)
        if kind == x_kind:  # in place
            B.relu_backward(d_h, codes, d_h)
            torch.cuda.synchronize()
            assert torch.equal(d_h, d_pre)


# ------------------------------------------------------------------------------------ gradient of the matrices
class Gradient:
    def __init__(self, B, counts, n_in, n_out, x_kind="e4m3", y_kind="bf16", pow2=True, seed=0):
        g = np.random.default_rng(seed + n_in + n_out + sum(counts))
        self.B, self.n_in, self.n_out, self.pow2 = B, n_in, n_out, pow2
        self.E, self.R = len(counts), int(sum(counts))
        x = (g.standard_normal((self.R, n_in)) * np.exp(g.standard_normal((self.R, 1)))).astype(np.float32)
        nb = -(-n_in // 128)
        self.x, self.x_s = O.quantize_rows(x, x_kind, pow2) if self.R else (np.zeros((0, nb * 128)), np.zeros((nb, 0), np.float32))
        self.offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.x_q, self.x_scale, self.offsets = dev(self.x, x_kind), dev(self.x_s), ints(self.offs)
        self.d_y = dev(g.standard_normal((self.R, n_out)) * np.exp(g.standard_normal((self.R, 1))), y_kind)
        self.terms = {(True, "bf16"): 1, (True, "f16"): 2, (True, "f32"): 3, (False, "bf16"): 3, (False, "f16"): 5, (False, "f32"): 6}[pow2, y_kind]
        self.most = max(counts) if counts else 0

    def run(self, out, add=None, stream=None, workspace=True):
        d_w = torch.full((self.E, self.n_in, self.n_out), 7.0, device="cuda").to(TORCH[out])
        need = self.B.expert_weight_gradient_workspace_bytes(self.R, self.E, self.n_in, self.n_out)
        ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda") if need and workspace else None
        self.B.expert_weight_gradient(self.x_q, self.x_scale, self.d_y, self.offsets, d_w, add, self.pow2, ws, stream)
        torch.cuda.synchronize()
        return d_w

    def check(self, out="f32", add=None, workspace=True):
        want, mag = O.expert_weight_gradient(self.x[:, :self.n_in], self.x_s, f64(self.d_y), self.offs, None if add is None else f64(add))
        got = self.run(out, add, workspace=workspace)
        # a product goes through at most one rounding a term of the sum, and there are `terms` for each row; parts of a sum and `add` are one more each.  Code times scale is
        # rounded once.  Pieces are cut off after 8 bits: the second is below 2^-7 of the value, the third below 2^-14, the three are the value but for 2^-32.  Left out are
        # second times third both ways and third times third: below 2 * 2^-21 + 2^-28 of the product, 17 H
        near(got, want, (self.terms * self.most + 16 + 1 + (17 if self.terms > 4 else 1)) * H * mag, out)
        return got


COUNTS = [[1], [0, 1, 0], [2, 0, 3], [0, 0, 0], [31, 0, 32, 33], [64, 65, 0, 63], [130, 1, 0, 257], [1] * 40, [600]]


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: "x".join(map(str, c[:6])))
@pytest.mark.parametrize("n_in,n_out", [(128, 128), (1, 1), (200, 300), (384, 517), (136, 264)])
def test_expert_weight_gradient(B, counts, n_in, n_out):
    say("gradient", counts[:6], n_in, n_out)
    for i, (pow2, y_kind) in enumerate([(p, y) for p in (True, False) for y in DTYPES]):
        p = Gradient(B, counts, n_in, n_out, "e5m2" if i % 2 else "e4m3", y_kind, pow2)
        for out in DTYPES if y_kind == "bf16" else ("f32",):
            p.check(out)


@pytest.mark.parametrize("counts,n_in,n_out,y_kind,pow2", [([700, 300], 1024, 640, "bf16", True), ([90] * 20, 768, 512, "bf16", True), ([4, 2, 0, 7] * 16, 512, 264, "f32", False),
                                                           ([2000, 0, 9], 256, 256, "bf16", True), ([1500], 300, 520, "f16", False), ([40] * 8, 512, 1024, "f16", True),
                                                           ([0, 2000, 1, 31, 64, 65, 700] + [150] * 9, 500, 2040, "bf16", True), ([0, 64, 1] + [300] * 13, 512, 2048, "bf16", True),
                                                           ([33] * 20, 520, 300, "f16", False), ([20, 0, 70] * 8, 300, 530, "f32", False), ([3000], 130, 200, "bf16", False),
                                                           ([0, 4000, 1, 20], 250, 252, "f32", True)])
def test_expert_weight_gradient_of_ordinary_sizes(B, counts, n_in, n_out, y_kind, pow2):
    say("gradient", counts[:6], n_in, n_out, y_kind, pow2)
    p = Gradient(B, counts, n_in, n_out, "e4m3", y_kind, pow2)
    p.check("f32")
    add = dev(np.random.default_rng(1).standard_normal((p.E, n_in, n_out)), "bf16")
    p.check("bf16", add)
    if B.expert_weight_gradient_workspace_bytes(p.R, p.E, n_in, n_out):
        p.check("f32", workspace=False)


@pytest.mark.parametrize("counts,n_in,n_out,y_kind,pow2", [([0, 900, 900, 40, 0, 300], 1000, 1300, "f32", False), ([0, 900, 900, 40, 0, 300], 1000, 1304, "f16", False),
                                                           ([5, 1500, 0, 1500, 64] + [100] * 7, 1040, 1304, "bf16", True), ([5, 1500, 0, 1500, 64] + [100] * 7, 1040, 1304, "bf16", False),
                                                           ([2100] + [1] * 7, 1152, 1288, "f16", False)])
def test_expert_weight_gradient_of_experts_of_very_different_size(B, counts, n_in, n_out, y_kind, pow2):
    """Items go by how many rows an expert has: two have as many, some none; each matrix is its own expert's."""
    say("gradient", counts[:6], n_in, n_out, y_kind, pow2)
    p = Gradient(B, counts, n_in, n_out, "e4m3", y_kind, pow2)
    got = p.check("f32")
    assert torch.equal(got, p.run("f32"))
    assert all(got[e].any() == (c > 0) for e, c in enumerate(counts))


@pytest.mark.parametrize("out", DTYPES)
@pytest.mark.parametrize("n_in,n_out", [(200, 136), (130, 77)])
def test_expert_weight_gradient_is_added(B, out, n_in, n_out):
    """To another tensor and in place; an expert without rows gives what is added."""
    say("gradient added", out, n_in, n_out)
    p = Gradient(B, [40, 0, 70], n_in, n_out)
    add = dev(np.random.default_rng(1).standard_normal((3, n_in, n_out)), out)
    got = p.check(out, add)
    assert torch.equal(got[1], add[1])
    ws = p.B.expert_weight_gradient_workspace_bytes(p.R, p.E, n_in, n_out)
    p.B.expert_weight_gradient(p.x_q, p.x_scale, p.d_y, p.offsets, add, add, True, torch.zeros(ws, dtype=torch.uint8, device="cuda") if ws else None)
    torch.cuda.synchronize()
    assert torch.equal(got, add)


def test_expert_weight_gradient_of_operands_with_strides(B):
    """Rows inside wider buffers, at addresses that wide loads do not reach, neighbours that are not finite, on another stream."""
    say("gradient strides")
    p = Gradient(B, [20, 0, 45, 130], 200, 136)
    want, mag = O.expert_weight_gradient(p.x[:, :200], p.x_s, f64(p.d_y), p.offs)
    wide = torch.full((p.R, 384 + 16), float("nan"), device="cuda").to(torch.float8_e4m3fn)
    wide[:, 16:16 + 256] = p.x_q
    p.x_q = wide[:, 16:16 + 256]
    scale = torch.full((2, p.R + 9), float("nan"), device="cuda")
    scale[:, 4:4 + p.R] = p.x_scale
    p.x_scale = scale[:, 4:4 + p.R]
    stream = torch.cuda.Stream()
    for at, width in ((8, 160), (3, 151)):
        d_y = torch.full((p.R, width), float("nan"), device="cuda").to(torch.bfloat16)
        d_y[:, at:at + 136] = p.d_y
        kept, p.d_y = p.d_y, d_y[:, at:at + 136]
        torch.cuda.synchronize()
        near(p.run("f32", stream=stream), want, (130 + 20) * H * mag, "f32")
        p.d_y = kept


def test_expert_weight_gradient_of_offsets_that_are_none(B):
    """Offsets outside the rows, or that fall, are taken as far as there are rows."""
    say("gradient offsets")
    p = Gradient(B, [50, 50], 130, 140)
    for offs in ([-5, 40, 2000], [60, 30, 90], [100, 100, 100], [-2 ** 31, 0, 2 ** 31 - 1]):
        p.offsets = ints(offs)
        got = p.run("f32")
        for e in range(2):
            lo = max(0, min(offs[e], p.R))
            hi = max(lo, min(offs[e + 1], p.R))
            want, mag = O.expert_weight_gradient(p.x[lo:hi, :130], p.x_s[:, lo:hi], f64(p.d_y)[lo:hi], [0, hi - lo])
            near(got[e:e + 1], want, (hi - lo + 20) * H * mag, "f32")


@pytest.mark.parametrize("pow2,y_kind", [(True, "bf16"), (True, "f16"), (True, "f32"), (False, "bf16"), (False, "f32")])
def test_expert_weight_gradient_passes_on_what_is_not_finite(B, pow2, y_kind):
    """To the row and column of the product it is in, and to no other expert: not from the rows behind an expert's last, which end in the middle of what is
    multiplied at once."""
    say("gradient not finite", pow2, y_kind)
    p = Gradient(B, [37, 20, 3], 136, 144, "e5m2", y_kind, pow2)
    finite = p.run("f32")
    d_y, x = p.d_y.clone(), p.x_q.clone()
    p.d_y[40, 7] = float("nan")            # expert 1
    p.d_y[57, 100] = float("inf")          # expert 2
    got = p.run("f32")
    assert torch.equal(got[0], finite[0])
    assert torch.isnan(got[1][:, 7]).all()
    keep = torch.ones(144, dtype=torch.bool, device="cuda")
    keep[7] = False
    assert torch.equal(got[1][:, keep], finite[1][:, keep])
    keep[7], keep[100] = True, False
    assert torch.equal(got[2][:, keep], finite[2][:, keep])
    xv = torch.from_numpy(p.x[57, :136]).cuda()
    assert torch.equal(got[2][:, 100] == float("inf"), xv > 0) and torch.equal(got[2][:, 100] == -float("inf"), xv < 0)
    p.d_y = d_y
    x[2, 5], x[59, 130] = float("nan"), float("-inf")
    p.x_q = x
    got = p.run("f32")
    assert torch.isnan(got[0][5]).all() and torch.equal(got[1], finite[1])
    rows = torch.arange(136, device="cuda")
    assert torch.equal(got[0][rows != 5], finite[0][rows != 5]) and torch.equal(got[2][rows != 130], finite[2][rows != 130])
    last = p.d_y[59].float()
    assert torch.equal(got[2][130] == -float("inf"), last > 0) and torch.equal(got[2][130] == float("inf"), last < 0)


def tiny(g, shape, lowest):
    """Float32 of 24 bits and of eight, magnitudes from 2^lowest to 2^(lowest + 60), each sign."""
    v = (1 + g.random(shape)) * np.exp2(g.integers(lowest, lowest + 60, shape))
    v = np.where(g.random(shape) < 0.5, v, np.exp2(np.floor(np.log2(v))))
    return (v * g.choice([-1, 1], shape)).astype(np.float32)


def keep_rows(p, x, x_kind, scale):
    """Rows x of codes' values, [R, n_in], with scales [blocks, R], in place of the ones p has."""
    p.x[:, :p.n_in], p.x_s = x, scale.astype(np.float32)
    p.x_q, p.x_scale = dev(p.x, x_kind), dev(p.x_s)
    p.x = f64(p.x_q)


@pytest.mark.parametrize("y_kind,x_kind,pow2", [("f32", "e5m2", True), ("f32", "e5m2", False), ("f32", "e4m3", False), ("bf16", "e4m3", False), ("f16", "e5m2", False)])
def test_expert_weight_gradient_of_tiny_values(B, y_kind, x_kind, pow2):
    """Next to infinities they count with their sign, however small they are, and among finite values they are off by a few of bfloat16's least steps, 2^-133: a
    value's three pieces are each a step from it at most, so an operand is below 2^-131 off."""
    say("gradient tiny", y_kind, x_kind, pow2)
    counts, n_in, n_out = [9, 0, 34], 136, 144
    p = Gradient(B, counts, n_in, n_out, x_kind, y_kind, pow2)
    g = np.random.default_rng(n_in)
    if y_kind == "f32":
        p.d_y = dev(tiny(g, (p.R, n_out), -149))
        assert (f64(p.d_y) != 0).all()
    if not pow2:
        small = (1 + g.random((2, p.R))) * np.exp2(g.integers(-126, -90, (2, p.R)))
        if y_kind == "f32":
            small = np.where(g.random((2, p.R)) < 0.5, small, 1 + g.random((2, p.R)))
        small[:, 3], small[:, 20] = 2.0 ** -126, 1.5 * 2.0 ** -115      # rows that meet an infinity below
        keep_rows(p, p.x[:, :n_in], x_kind, small)
    for finite in (True, False):
        if not finite:
            d_y, x = f64(p.d_y), p.x.copy()
            d_y[3, 5], d_y[20, 100] = np.inf, -np.inf
            p.d_y = dev(d_y, y_kind)
            if x_kind == "e5m2":
                x[7, 11], x[30, 130] = -np.inf, np.inf
                keep_rows(p, x[:, :n_in], x_kind, p.x_s)
        got = f64(p.run("f32"))
        with np.errstate(invalid="ignore"):
            want, mag = O.expert_weight_gradient(p.x[:, :n_in], p.x_s, f64(p.d_y), p.offs)
        there = np.isfinite(want)
        assert there.all() == finite
        same = np.array_equal(got[~there], want[~there], equal_nan=True)
        assert same, finite
        xs = np.abs(p.x[:, :n_in] * np.repeat(p.x_s.astype(np.float64).T, 128, axis=1)[:, :n_in])
        for e in range(3):
            lo, hi = p.offs[e], p.offs[e + 1]
            # relative as for other values; an operand off by 2^-131 beside the other's magnitude, twice as much for the products that are left out; sums below 2^-126 are multiples
            # of 2^-149 after each of their terms; code times scale is one in float32
            with np.errstate(invalid="ignore"):
                err = (p.terms * 34 + 34) * H * mag[e] + 2.0 ** -130 * (xs[lo:hi].sum(0)[:, None] + np.abs(f64(p.d_y)[lo:hi]).sum(0)[None]) + p.terms * 34 * 2.0 ** -149
                assert np.all(np.abs(got[e] - want[e])[there[e]] <= err[there[e]]), (e, finite)


@pytest.mark.parametrize("y_kind", DTYPES)
@pytest.mark.parametrize("x_kind,pow2,scale,least", [("e4m3", True, 2.0 ** -126, 2.0 ** -134), ("e4m3", True, 2.0 ** -124, 0), ("e4m3", True, 2.0 ** 120, 0), ("e5m2", True, 2.0 ** -126, 2.0 ** -134),
                                                     ("e5m2", True, 2.0 ** -117, 0), ("e5m2", True, 2.0 ** 112, 0), ("e4m3", False, 1.25 * 2.0 ** -126, 2.0 ** -131), ("e5m2", False, 2.0 ** -126, 2.0 ** -131),
                                                     ("e4m3", False, 1.9 * 2.0 ** 119, 2.0 ** -131), ("e5m2", False, 1.9 * 2.0 ** 111, 2.0 ** -131)])
def test_expert_weight_gradient_at_both_ends_of_the_scales(B, x_kind, pow2, scale, least, y_kind):
    """Every finite code but those that the scale takes past float32.  `least`: how far an operand may be off besides roundings: half of bfloat16's least step where a scale that is a power
    of two leaves less than that, and 2^-131 for three pieces."""
    say("gradient scales", x_kind, pow2, scale, y_kind)
    counts, n_in, n_out = [300], 136, 144
    p = Gradient(B, counts, n_in, n_out, x_kind, y_kind, pow2)
    codes = torch.arange(256, dtype=torch.uint8).view(TORCH[x_kind]).float().double().numpy()
    codes = codes[np.isfinite(codes) & (np.abs(codes * scale) < 2.0 ** 127)]
    g = np.random.default_rng(int(n_in + abs(np.log2(scale))))
    keep_rows(p, g.choice(codes, (p.R, n_in)), x_kind, np.full((2, p.R), scale))
    p.d_y = dev(g.standard_normal((p.R, n_out)) * (2.0 ** -14 if scale > 1 else 1), y_kind)
    want, mag = O.expert_weight_gradient(p.x[:, :n_in], p.x_s, f64(p.d_y), p.offs)
    y = np.abs(f64(p.d_y)).sum(0)
    # gradients of three pieces are 2^-131 off beside a code times its scale; sums below 2^-126 are multiples of 2^-149 after each of their terms; (-0 and 0 in `codes` make zeros)
    x = np.abs(p.x[:, :n_in]).sum(0)[:, None] * scale
    err = (p.terms * p.R + 34) * H * mag + least * y[None] + (2.0 ** -130 * x if y_kind == "f32" else 0) + p.terms * p.R * 2.0 ** -149
    got = f64(p.run("f32"))
    assert np.isfinite(got).all() and np.abs(want).max() < 2.0 ** 126
    worst = (np.abs(got - want) - err).max()
    assert worst <= 0
    if scale < 1:
        assert got.any()


@pytest.mark.parametrize("y_kind", DTYPES)
def test_expert_weight_gradient_of_rows_with_a_scale_of_zero(B, y_kind):
    """Codes that are left over in rows whose scales are 0, which a plan's spare rows are cleared to, add nothing: the bits of zero codes."""
    say("gradient scales of zero", y_kind)
    p = Gradient(B, [60, 7], 136, 144, "e4m3", y_kind, False)
    p.x_scale[:, 10:20] = 0
    p.x_scale[1, 60:] = 0
    got = p.run("f32")
    codes = p.x_q.view(torch.uint8)
    codes[10:20] = 0
    codes[60:, 128:] = 0
    assert torch.equal(got, p.run("f32")) and not got[1][128:].any() and got[1][:128].any()


def test_expert_weight_gradient_is_that_of_differences_of_the_product(B):
    """The loss <x . W, c> of expert_matmul is linear in W: for a W of one code the product is that entry's column of x times it."""
    say("gradient differences")
    g = np.random.default_rng(6)
    counts, n_in, n_out = [9, 0, 50], 200, 140
    E, R = len(counts), sum(counts)
    offs = ints(np.concatenate([[0], np.cumsum(counts)]))
    xq, xs = codes_for(R, n_in, "e4m3")
    B.quantize_rows(dev(g.standard_normal((R, n_in))), xq, xs, pow2=True)
    c = dev(g.standard_normal((R, n_out)), "bf16")
    d_w = torch.zeros(E, n_in, n_out, device="cuda")
    B.expert_weight_gradient(xq, xs, c, offs, d_w, pow2=True)
    qs, ss = B.fp8_weight_shapes(E, n_in, n_out)
    for e, i, o in ((0, 0, 0), (2, 150, 139), (2, 199, 64), (1, 3, 3)):
        w = torch.zeros(E, n_in, n_out, device="cuda")
        w[e, i, o] = 448.0
        wq, ws = torch.zeros(qs, device="cuda").to(torch.float8_e4m3fn), torch.zeros(ss, device="cuda")
        B.quantize_weights(w, wq, ws)
        y = torch.zeros(R, n_out, device="cuda")
        B.expert_matmul(xq, xs, wq, ws, offs, n_in, n_out, y)
        torch.cuda.synchronize()
        terms = f64(y) * f64(c) / 448
        assert abs(terms.sum() - f64(d_w)[e, i, o]) <= (50 + 20) * H * np.abs(terms).sum()


def test_expert_weight_gradient_with_offsets_that_pass_32_bits(B):
    """Rows of gradients and codes, and results, beyond the first 4 GiB of their buffers."""
    say("gradient 32 bits")
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of memory")
    R, E, n_in, n_out = 300, 3, 130, 136
    p = Gradient(B, [100, 50, 150], n_in, n_out)
    d_y = torch.empty(R * (1 << 23), dtype=torch.bfloat16, device="cuda").as_strided((R, n_out), (1 << 23, 1))      # 5 GB
    d_y.copy_(p.d_y)
    x = torch.empty(R * (1 << 24), dtype=torch.uint8, device="cuda").as_strided((R, 256), (1 << 24, 1)).view(torch.float8_e4m3fn)  # 5 GB
    x.view(torch.uint8).copy_(p.x_q.view(torch.uint8))
    want = p.run("f32")
    p.d_y, p.x_q = d_y, x
    assert torch.equal(p.run("f32"), want)
    del d_y, x
    p = Gradient(B, [1, 2] + [0] * 248 + [3], 4096, 4104)       # 4.2 G results
    got = p.run("bf16")
    last, mag = O.expert_weight_gradient(p.x[3:, :4096], p.x_s[:, 3:], f64(p.d_y)[3:], [0, 3])
    near(got[250:], last, 23 * H * mag, "bf16")
    assert not got[249].any() and not got[100].any()


def test_dispatch_and_combine_with_offsets_that_pass_32_bits(B):
    say("rows 32 bits")
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of memory")
    T, d = 300, 136
    g = np.random.default_rng(2)
    x = dev(g.standard_normal((T, d)), "bf16")
    rows = torch.empty(T * (1 << 23), dtype=torch.bfloat16, device="cuda").as_strided((T, d), (1 << 23, 1))
    row_of = g.permutation(T).astype(np.int32)
    B.dispatch_rows(x, ints(row_of), rows)
    y, d_w = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, 1, device="cuda")
    B.combine_rows(rows, ints(row_of), y)
    B.combine_rows_backward(x, rows, ints(row_of), None, None, d_w)
    torch.cuda.synchronize()
    assert torch.equal(y, x)
    xs = f64(x)
    near(d_w[:, 0], (xs * xs).sum(1), 17 * H * (xs * xs).sum(1), "f32")


@pytest.mark.parametrize("at,width", [(1, 140), (3, 151), (8, 160), (4, 148)])
@pytest.mark.parametrize("kind", DTYPES)
def test_rows_inside_wider_buffers(B, kind, at, width):
    """Rows of every call at addresses that nothing but the type aligns: the bits of rows that lie side by side, and neighbours stay as they are."""
    say("strides", kind, at, width)
    g = np.random.default_rng(at)
    T, k, d = 1100, 2, 131 if at % 2 else 136
    row_of, R = entries(g, T, k, dropped=100)
    of, w = ints(row_of), dev(g.random((T, k)))

    def wide(t):
        b = torch.full((t.shape[0], width), float("nan"), device="cuda").to(t.dtype)
        b[:, at:at + d] = t
        return b[:, at:at + d], b

    def alike(view, buffer, want):
        torch.cuda.synchronize()
        assert torch.equal(view, want)
        buffer[:, at:at + d] = float("nan")
        assert torch.isnan(buffer).all()
    x, rows = dev(g.standard_normal((T, d)), kind), dev(g.standard_normal((R, d)), kind)
    h = torch.from_numpy(g.integers(0, 256, (R, 256)).astype(np.uint8)).cuda().view(torch.float8_e4m3fn)
    (xw, _), (rw, _) = wide(x), wide(rows)
    for q_kind in (None, "e5m2"):
        codes = lambda: codes_for(R, d, q_kind) if q_kind else (None, None)  # noqa: E731
        same = lambda a, b: q_kind is None or (torch.equal(a[0].view(torch.uint8), b[0].view(torch.uint8)) and torch.equal(a[1], b[1]))  # noqa: E731
        for call in (lambda x, r, o, c: B.dispatch_rows(x, of, o, *c, weight=w), lambda x, r, o, c: B.relu_backward(r, h, o, *c)):
            out, c, cw = torch.full_like(rows, 7.0), codes(), codes()
            call(x, rows, out, c)
            o, buffer = wide(torch.full_like(rows, 7.0))
            call(xw, rw, o, cw)
            alike(o, buffer, out)
            assert same(c, cw)
        out, c, cw, d_w, d_ww = torch.full_like(rows, 7.0), codes(), codes(), torch.zeros(T, k, device="cuda"), torch.ones(T, k, device="cuda")
        B.combine_rows_backward(x, rows, of, w, out, d_w, *c)
        o, buffer = wide(torch.full_like(rows, 7.0))
        B.combine_rows_backward(xw, rw, of, w, o, d_ww, *cw)
        alike(o, buffer, out)
        assert same(c, cw) and torch.equal(d_w, d_ww)
    out = torch.full_like(x, 7.0)
    B.combine_rows(rows, of, out, w, x)
    o, buffer = wide(torch.full_like(x, 7.0))
    B.combine_rows(rw, of, o, w, xw)
    alike(o, buffer, out)


def test_first_call_of_a_kernel_inside_a_capture(B):
    """A kernel with more LDS than a launch gets by itself, run for the first time in this process while a graph is captured."""
    say("first call captured")
    p = Gradient(B, [3, 0, 40], 130, 100, "e5m2", "f32", False)
    d_w = torch.zeros(3, 130, 100, device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        B.expert_weight_gradient(p.x_q, p.x_scale, p.d_y, p.offsets, d_w, stream=stream)
    for _ in range(3):
        d_w.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(d_w, p.run("f32"))
    del graph


@pytest.mark.parametrize("T,k,d", [(1100, 2, 520), (1030, 3, 1000), (1025, 2, 1024), (1100, 2, 1216), (1100, 2, 1217), (1026, 3, 1999), (1027, 2, 2056), (1040, 2, 4099), (1030, 2, 4616)])
def test_many_tokens_of_long_rows(B, T, k, d):
    """More than 1024 tokens: a wavefront goes through one, two or four times 512 columns at once, the last of which may be there in part or not at all, and comes back for
    more; entries of one wavefront each, also where rows lie anywhere."""
    say("many tokens", T, k, d)
    g = np.random.default_rng(d)
    row_of, R = entries(g, T, k, dropped=T // 3, spare=3)
    of, w = ints(row_of), g.standard_normal((T, k)).astype(np.float32)
    for r_kind, kind in (("bf16", "bf16"), ("f32", "f16"), ("f16", "f32")):
        rows, add = dev(g.standard_normal((R, d)), r_kind), dev(g.standard_normal((T, d)), kind)
        for weight, added in ((w, add), (None, None)):
            y = torch.full((T, d), 7.0, device="cuda").to(TORCH[kind])
            B.combine_rows(rows, of, y, None if weight is None else dev(weight), added)
            torch.cuda.synchronize()
            want, mag = O.combine_rows(f64(rows), row_of, T, weight, None if added is None else f64(added))
            near(y, want, (k + 1) * H * mag, kind)
            if added is not None:
                B.combine_rows(rows, of, add, dev(w), add)
                torch.cuda.synchronize()
                assert torch.equal(add, y)
    for x_kind, kind, q_kind, pow2 in (("bf16", "bf16", "e5m2", False), ("f32", "f16", "e4m3", d < 1300), ("bf16", "f32", None, False)):
        d_y, rows = dev(g.standard_normal((T, d)), x_kind), dev(g.standard_normal((R, d)), kind)
        want = O.dispatch_rows(f64(d_y), row_of, R, w)
        named = ~np.isnan(want[:, 0])
        want_w, mag = O.combine_weight_gradient(f64(d_y), f64(rows), row_of)
        for backward in (True, False):
            out, (q, s), d_w = torch.full_like(rows, 7.0), codes_for(R, d, q_kind) if q_kind else (None, None), torch.full((T, k), 7.0, device="cuda")
            if backward:
                B.combine_rows_backward(d_y, rows, of, dev(w), out, d_w, q, s, pow2)
            else:
                B.dispatch_rows(d_y, of, out, q, s, dev(w), pow2)
            torch.cuda.synchronize()
            near(f64(out)[named], want[named], H * np.abs(want[named]) + 2.0 ** -150, kind)
            assert np.all(f64(out)[~named] == 7)
            if q_kind:
                check_codes(q, s, np.nan_to_num(want), d, q_kind, pow2, named)
            if backward:  # a lane's products one after the other, six sums over the lanes, three over the wavefronts
                near(d_w, want_w, (8 * -(-d // 512) + 9) * H * mag + 2.0 ** -140, "f32")


CAPTURED_FIRST = """
import torch
from paper_2308_12066_amd import binding as B
g = torch.Generator(device="cuda").manual_seed(1)
R, E, n_in, n_out = 43, 3, 130, 100
x = torch.randn(R, 256, generator=g, device="cuda").to(torch.float8_e5m2)
scale, d_y = torch.rand(2, R, generator=g, device="cuda") + 0.5, torch.randn(R, n_out, generator=g, device="cuda")
offsets = torch.tensor([0, 3, 3, R], dtype=torch.int32, device="cuda")
d_w, eager = (torch.full((E, n_in, n_out), 7.0, device="cuda") for _ in range(2))
stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph, stream=stream):
    B.expert_weight_gradient(x, scale, d_y, offsets, d_w, stream=stream)
for _ in range(3):
    d_w.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    B.expert_weight_gradient(x, scale, d_y, offsets, eager)
    torch.cuda.synchronize()
    assert torch.equal(d_w, eager) and not d_w[1].any() and d_w[0].any() and d_w[2].any()
del graph
print("replays give the eager bits")
"""


def test_first_call_of_a_kernel_in_a_process_may_be_captured():
    """One with more LDS than a launch gets by itself, in a process that has run none before: the limit is raised while a graph is captured."""
    import os
    import subprocess
    import sys
    say("first call captured, process of its own")
    child = subprocess.run([sys.executable, "-c", CAPTURED_FIRST], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=100)
    assert child.returncode == 0 and "eager bits" in child.stdout, child.stderr[-2000:]


def test_no_call_of_training_allocates(B):
    """All five, after the first time, which loads them: a buffer of any of their results would be more than what is allowed for."""
    say("training, memory")
    g = np.random.default_rng(4)
    T, k, d, f, counts = 8000, 2, 1100, 640, [9000, 0, 7000]
    row_of, R = entries(g, T, k)
    of, offs, w = ints(row_of), ints(np.concatenate([[0], np.cumsum(counts)])), dev(g.random((T, k)))
    x, rows, d_h, d_w, d_weight = torch.randn(T, d, device="cuda"), torch.zeros(R, d, device="cuda"), torch.randn(R, f, device="cuda"), torch.zeros(3, d, f, device="cuda"), torch.zeros(T, k, device="cuda")
    y, d_rows, d_pre, (q, s), (h, _), (p, ps) = torch.zeros_like(x), torch.zeros_like(rows), torch.zeros_like(d_h), codes_for(R, d, "e4m3"), codes_for(R, f, "e5m2"), codes_for(R, f, "e5m2")
    need = B.expert_weight_gradient_workspace_bytes(R, 3, d, f)
    ws = torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda")

    def step():
        B.dispatch_rows(x, of, rows, q, s, w)
        B.combine_rows(rows, of, y, w, x)
        B.combine_rows_backward(x, rows, of, w, d_rows, d_weight, q, s)
        B.relu_backward(d_h, h, d_pre, p, ps)
        B.expert_weight_gradient(q, s, d_h, offs, d_w, d_w, False, ws)
    step()
    torch.cuda.synchronize()
    free, held = torch.cuda.mem_get_info()[0], torch.cuda.memory_allocated()
    for _ in range(3):
        step()
    now = torch.cuda.mem_get_info()[0]      # while the calls may still run
    torch.cuda.synchronize()
    # (torch's share may fall: what an earlier test left in a cycle goes at any time)
    assert min(now, torch.cuda.mem_get_info()[0]) >= free - (4 << 20) and torch.cuda.memory_allocated() <= held


# ------------------------------------------------------------------------------------ together
@pytest.fixture(scope="module")
def example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "fp8_experts.py")
    spec = importlib.util.spec_from_file_location("fp8_experts", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("train", [False, True])
@pytest.mark.parametrize("T,d,f,E,k", [(1, 256, 512, 8, 2), (60, 128, 300, 16, 3), (400, 256, 520, 4, 2)])
def test_gradients_of_the_matrices_of_a_block(example, T, d, f, E, k, train):
    """Of examples/fp8_experts.py, against the chain in 64 bits from what the forward left and the calls' own 16-bit gradients' definition."""
    say("block gradients", T, d, f, E, k, train)
    g = np.random.default_rng(T)
    w1, w2 = ((0.05 * g.standard_normal(s)).astype(np.float32) for s in ((E, d, f), (E, f, d)))
    x, z, dy = dev(g.standard_normal((T, d)), "bf16"), dev(g.standard_normal((T, E))), g.standard_normal((T, d)).astype(np.float32)
    block = example.Block(dev(w1), dev(w2), None, k, T, train=train, renormalize=True)
    block.forward(x, z)
    without = block.backward(z, dev(dy))
    start = [dev(g.standard_normal(s)) for s in ((E, d, f), (E, f, d))]
    d_w = [t.clone() for t in start]
    with_them = block.backward(z, dev(dy), d_w=d_w)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(without, with_them))
    row_of, offs, wt = block.row_of.cpu().numpy(), block.offsets.cpu().numpy(), f64(block.weight)
    d_rows = np.nan_to_num(O.dispatch_rows(dy.astype(np.float64), row_of, T * k, wt.astype(np.float32)))
    x_q, h_q = f64(block.x_q[0])[:, :d], f64(block.h_q[0])[:, :f]
    x_s, h_s = f64(block.x_q[1]), f64(block.h_q[1])
    if train:
        assert np.all(np.frexp(x_s)[0] == 0.5) and np.all(np.frexp(h_s)[0] == 0.5)
    most = int(np.diff(offs).max())
    want, mag = O.expert_weight_gradient(h_q, h_s, d_rows, offs, f64(start[1]))
    # gradients of the rows rounded to bfloat16, 2^-8 of each, then the product's roundings (three for each row at most)
    near(d_w[1], want, (2.0 ** -8 * (1 + H) + (3 * most + 20) * H) * mag, "f32")
    qv, qs = O.quantize_rows(d_rows.astype(np.float32), "e5m2")
    q2, s2 = O.quantize_weights(w2)
    d_h, d_h_mag = O.expert_matmul(qv[:, :d], qs, q2.transpose(0, 2, 1), s2.transpose(0, 2, 1), offs)
    d_pre = O.relu_backward(d_h, h_q)
    want, mag = O.expert_weight_gradient(x_q, x_s, d_pre, offs, f64(start[0]))
    _, off = O.expert_weight_gradient(x_q, x_s, np.where(h_q > 0, (128 + 4 * -(-d // 128)) * H * d_h_mag, 0), offs)      # what the product before may be off
    near(d_w[0], want, (2.0 ** -8 * (1 + H) + (3 * most + 20) * H) * (mag + off) + off, "f32")
    block.close()


def test_gradients_of_a_block_take_a_gradient_that_lies_in_any_way(example):
    """One row for all tokens (what the sum over tokens has for a gradient), one number for all, columns that do not lie side by side: the bits of a copy."""
    say("block gradients, layouts")
    T, d, f, E, k = 50, 128, 200, 8, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    block = example.Block(0.05 * normal(E, d, f), 0.05 * normal(E, f, d), None, k, T, train=True, renormalize=True)
    x, z = normal(T, d).bfloat16(), normal(T, E)
    block.forward(x, z)
    for d_y in (normal(1, d).expand(T, d), normal(1, 1).expand(T, d), normal(d, T).t(), normal(T, 2 * d)[:, ::2]):
        both = []
        for t in (d_y, d_y.clone(memory_format=torch.contiguous_format)):
            d_w = torch.zeros(E, d, f, device="cuda"), torch.zeros(E, f, d, device="cuda")
            both.append([*block.backward(z, t, d_w=d_w), *d_w])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*both))
    block.close()


def test_step_of_training_replays_from_a_captured_graph(example):
    """Forward, backward and gradients of the matrices of a block, captured; replays with the eager work of other inputs between them give the eager bits."""
    say("training captured")
    T, d, f, E, k = 96, 128, 260, 8, 2
    g = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    w1, w2 = 0.05 * normal(E, d, f), 0.05 * normal(E, f, d)
    block = example.Block(w1, w2, None, k, T, train=True, renormalize=True)
    x, z, dy, d_w = normal(T, d).bfloat16(), normal(T, E), normal(T, d), (torch.zeros(E, d, f, device="cuda"), torch.zeros(E, f, d, device="cuda"))
    inputs = [(normal(T, d).bfloat16(), normal(T, E), normal(T, d)) for _ in range(3)]

    def step(stream=None):
        return block.forward(x, z, stream), *block.backward(z, dy, stream, d_w=d_w)

    def put(values):
        for to, of in zip((x, z, dy), values):
            to.copy_(of)
        for t in d_w:
            t.zero_()
        torch.cuda.synchronize()

    eager = []
    for values in inputs:
        put(values)
        eager.append([t.clone() for t in (*step(), *d_w)])
        torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outputs = step(stream)
    for rep in range(3):
        for values, want in zip(inputs, eager):
            put(values)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((*outputs, *d_w), want)), rep
            put(inputs[rep])
            step()
            torch.cuda.synchronize()
    del graph
    block.close()


def test_training_calls_on_another_stream_behind_what_fills_their_inputs(B):
    """Torch's current stream is another than the default one and busy: each call waits for its inputs, and torch for it."""
    say("training stream")
    g = np.random.default_rng(2)
    T, k, d, n_out, counts = 64, 2, 200, 136, [50, 0, 78]
    row_of, R = entries(g, T, k)
    x, w, of, offs = dev(g.standard_normal((T, d))), dev(g.random((T, k))), ints(row_of), ints(np.concatenate([[0], np.cumsum(counts)]))
    d_y = dev(g.standard_normal((R, n_out)), "bf16")

    def run(x, w, d_y):
        rows, y, d_w, d_rows = (torch.zeros(s, device="cuda") for s in ((R, d), (T, d), (T, k), (R, d)))
        q, s = codes_for(R, d, "e4m3")
        B.dispatch_rows(x, of, rows, q, s, w, pow2=True)
        B.combine_rows(rows, of, y, w)
        B.combine_rows_backward(y, rows, of, w, d_rows, d_w)
        d_pre = torch.zeros(R, d, device="cuda")
        B.relu_backward(d_rows, q, d_pre)
        grad = torch.zeros(3, d, n_out, device="cuda")
        B.expert_weight_gradient(q, s, d_y, offs, grad, pow2=True)
        return [t.clone() for t in (rows, y, d_w, d_rows, d_pre, grad)]
    want = run(x, w, d_y)
    torch.cuda.synchronize()
    late = [torch.zeros_like(t) for t in (x, w, d_y)]
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(3):
            big = big @ big * 1e-4                           # some milliseconds
        for to, t in zip(late, (x, w, d_y)):
            to.copy_(t)
        got = run(*late)
        torch.cuda.current_stream().synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_calls_of_training_leave_the_devices_memory_alone(B):
    """No call allocates, and the same call twice gives the same bits."""
    say("training bits")
    g = np.random.default_rng(9)
    p = Gradient(B, [5000, 0, 40], 200, 264)
    assert B.expert_weight_gradient_workspace_bytes(p.R, p.E, p.n_in, p.n_out) > 0
    first = p.run("f32")
    for _ in range(3):
        assert torch.equal(p.run("f32"), first)
    need = B.expert_weight_gradient_workspace_bytes(p.R, p.E, p.n_in, p.n_out)
    for size in (need - 4, need, need + 400):       # with too small a workspace: without one
        ws = torch.full((size + 256,), 0xff, dtype=torch.uint8, device="cuda")
        d_w = torch.zeros(p.E, p.n_in, p.n_out, device="cuda")
        B.expert_weight_gradient(p.x_q, p.x_scale, p.d_y, p.offsets, d_w, None, True, ws[:size])
        torch.cuda.synchronize()
        assert torch.equal(d_w, first if size >= need else p.run("f32", workspace=False)) and torch.all(ws[size:] == 0xff)
        if size < need:
            assert torch.all(ws == 0xff)
    T, d = 3000, 300
    row_of, R = entries(g, T, 2)
    x, rows = dev(g.standard_normal((T, d))), dev(g.standard_normal((R, d)))
    d_w = [torch.zeros(T, 2, device="cuda") for _ in range(2)]
    free = torch.cuda.mem_get_info()[0]
    for t in d_w:
        B.combine_rows_backward(x, rows, ints(row_of), None, None, t)
    torch.cuda.synchronize()
    assert torch.equal(*d_w) and torch.cuda.mem_get_info()[0] >= free - (4 << 20)
