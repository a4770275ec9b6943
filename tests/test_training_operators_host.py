"""The operators that train a block of experts, without a GPU: what the entry points refuse, that correct arguments get as far as the
missing device, where the binding launches, and the plain 64-bit forms against hand-made values and differences."""
from ctypes import byref

import numpy as np
import pytest

from oracle import operators as O
from paper_2308_12066_amd import binding as B

torch = pytest.importorskip("torch")

BUF = np.zeros(1 << 16, dtype=np.uint8)
P = BUF.ctypes.data + (-BUF.ctypes.data) % 256      # aligned host memory standing in for device pointers
needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="a launch would go through")
POW2 = B.SCALE_POW2


def rows8(**kw):
    base = dict(q=P, q_stride=256, scale=P, scale_stride=8, rows=8, cols=200, dtype=B.E5M2)
    base.update(kw)
    return B.FP8Rows(**base)


def refused(rc, word):
    assert rc == B.EINVAL, (rc, B.last_error())
    assert word in B.last_error(), B.last_error()


DISPATCH = dict(x=P, x_stride=200, x_dtype=B.BF16, T=4, d=200, row_of=P, copies=2, weight=P, rows=P, rows_stride=200, rows_dtype=B.F32, n_rows=8, q=rows8())
COMBINE = dict(rows=P, rows_stride=200, rows_dtype=B.BF16, n_rows=8, row_of=P, copies=2, weight=P, add=P, add_stride=200, T=4, d=200, y=P, y_stride=200, y_dtype=B.F16)
BACKWARD = dict(d_y=P, d_y_stride=200, d_y_dtype=B.F32, T=4, d=200, rows=P, rows_stride=200, rows_dtype=B.BF16, n_rows=8, row_of=P, copies=2, weight=P, d_rows=P, d_rows_stride=200,
                q=rows8(), d_weight=P)
RELU = dict(d_h=P, d_h_stride=200, d_h_dtype=B.F32, rows=8, cols=200, h_q=P, h_q_stride=256, h_dtype=B.E4M3, d_pre=P, d_pre_stride=200, d_pre_dtype=B.BF16, q=rows8())
GRADIENT = dict(x=rows8(dtype=B.E4M3), d_y=P, d_y_stride=300, d_y_dtype=B.BF16, offsets=P, n_experts=4, n_out=300, add=P, d_w=P, d_w_dtype=B.F32, workspace=None, bytes=0)
CALLS = {"dispatch": ("pgmoe_dispatch_rows", DISPATCH), "combine": ("pgmoe_combine_rows", COMBINE), "backward": ("pgmoe_combine_rows_backward", BACKWARD),
         "relu": ("pgmoe_relu_backward", RELU), "gradient": ("pgmoe_expert_weight_gradient", GRADIENT)}


def call(which, **kw):
    name, base = CALLS[which]
    assert set(kw) <= set(base)
    return getattr(B.lib, name)(*[byref(v) if isinstance(v, B.FP8Rows) else v for v in dict(base, **kw).values()], None)


BAD = [
    ("dispatch", dict(T=-1), "T=-1"), ("dispatch", dict(copies=0), "copies=0"), ("dispatch", dict(d=0), "d=0"), ("dispatch", dict(d=(1 << 22) + 1), "d="),
    ("dispatch", dict(n_rows=-1), "n_rows"), ("dispatch", dict(T=1 << 25, copies=2), "launch"), ("dispatch", dict(T=(1 << 31) - 1, copies=(1 << 31) - 1), "launch"), ("dispatch", dict(T=(1 << 26) - 3, copies=1), "launch"), ("dispatch", dict(x_dtype=B.E4M3), "x_dtype"),
    ("dispatch", dict(rows_dtype=9), "rows_dtype"), ("dispatch", dict(x=None), "x is NULL"), ("dispatch", dict(x=P + 1), "x is not"), ("dispatch", dict(x_stride=199), "x has rows"),
    ("dispatch", dict(rows=P + 2), "rows is not"), ("dispatch", dict(rows_stride=199), "rows has rows"), ("dispatch", dict(row_of=None), "row_of is NULL"),
    ("dispatch", dict(row_of=P + 2), "row_of"), ("dispatch", dict(weight=P + 2), "weight"), ("dispatch", dict(rows=None, q=None), "both"),
    ("dispatch", dict(q=rows8(cols=190)), "rows_q is"), ("dispatch", dict(q=rows8(rows=7)), "rows_q is"), ("dispatch", dict(q=rows8(dtype=B.F32)), "dtype"),
    ("dispatch", dict(q=rows8(dtype=B.E4M3 | 0x200)), "dtype"), ("dispatch", dict(q=rows8(q=None)), "NULL"), ("dispatch", dict(q=rows8(q_stride=240)), "q_stride"),
    ("combine", dict(T=-1), "T=-1"), ("combine", dict(copies=0), "copies=0"), ("combine", dict(d=0), "d=0"), ("combine", dict(n_rows=-1), "n_rows"),
    ("combine", dict(T=1 << 25, copies=2), "launch"), ("combine", dict(rows_dtype=B.E5M2), "rows_dtype"), ("combine", dict(y_dtype=-1), "y_dtype"),
    ("combine", dict(rows=None), "rows is NULL"), ("combine", dict(rows_stride=100), "rows has"), ("combine", dict(add=P + 1), "add is not"),
    ("combine", dict(add_stride=100), "add has"), ("combine", dict(y=None), "y is NULL"), ("combine", dict(y_stride=199), "y has"), ("combine", dict(row_of=None), "row_of"),
    ("combine", dict(weight=P + 1), "weight"),
    ("backward", dict(T=-1), "T=-1"), ("backward", dict(copies=-2), "copies"), ("backward", dict(T=1 << 25, copies=2), "launch"), ("backward", dict(d_y_dtype=B.E4M3), "d_y_dtype"),
    ("backward", dict(rows_dtype=B.E4M3), "rows_dtype"), ("backward", dict(d_y=None), "d_y is NULL"), ("backward", dict(rows=None), "rows is NULL"),
    ("backward", dict(rows_stride=1), "rows has"), ("backward", dict(d_rows=P + 1), "d_rows is not"), ("backward", dict(d_rows_stride=1), "d_rows has"),
    ("backward", dict(d_rows=None, q=None, d_weight=None), "d_weight are NULL"), ("backward", dict(d_weight=P + 2), "d_weight"), ("backward", dict(q=rows8(rows=9, scale_stride=9)), "d_rows_q is"),
    ("backward", dict(row_of=None), "row_of"), ("backward", dict(weight=P + 2), "weight"),
    ("relu", dict(rows=-1), "rows"), ("relu", dict(cols=0), "columns"), ("relu", dict(d_h_dtype=B.E4M3), "d_h_dtype"), ("relu", dict(d_pre_dtype=B.E4M3), "d_pre_dtype"),
    ("relu", dict(d_h=None), "d_h is NULL"), ("relu", dict(d_h_stride=199), "d_h has"), ("relu", dict(h_q=None), "h_q"), ("relu", dict(h_q=P + 8), "h_q"),
    ("relu", dict(h_q_stride=128), "q_stride"), ("relu", dict(h_dtype=B.BF16), "h_q has dtype"), ("relu", dict(d_pre=None, q=None), "both"), ("relu", dict(d_pre_stride=1), "d_pre has"),
    ("relu", dict(q=rows8(cols=100)), "d_pre_q is"), ("relu", dict(rows=(1 << 31) - 1, cols=1 << 22, d_h_stride=1 << 22, h_q_stride=1 << 22, d_pre_stride=1 << 22, q=None), "launch"),
    ("gradient", dict(x=None), "x is NULL"), ("gradient", dict(x=rows8(dtype=B.BF16)), "dtype"), ("gradient", dict(x=rows8(scale=None)), "NULL"),
    ("gradient", dict(x=rows8(rows=(1 << 24) + 1, scale_stride=1 << 25)), "2^24"), ("gradient", dict(d_y_dtype=B.E5M2), "d_y_dtype"), ("gradient", dict(d_w_dtype=B.E5M2), "d_w_dtype"),
    ("gradient", dict(n_experts=0), "n_experts"), ("gradient", dict(n_experts=257), "n_experts"), ("gradient", dict(n_out=0), "n_out"), ("gradient", dict(n_out=(1 << 22) + 1), "n_out"),
    ("gradient", dict(d_y_stride=299), "d_y_stride"), ("gradient", dict(d_y=None), "d_y is NULL"), ("gradient", dict(d_y=P + 1), "d_y is not"), ("gradient", dict(offsets=None), "expert_offsets"),
    ("gradient", dict(d_w=None), "d_w is NULL"), ("gradient", dict(d_w=P + 2), "d_w is not"), ("gradient", dict(add=P + 2), "add is not"),
    ("gradient", dict(x=rows8(cols=1 << 22, q_stride=1 << 22), n_out=1 << 20, d_y_stride=1 << 20), "launch"), ("gradient", dict(workspace=P + 8, bytes=64), "workspace"),
]


@pytest.mark.parametrize("which,bad,word", BAD, ids=lambda v: v if isinstance(v, str) else ",".join(v))
def test_bad_arguments_are_refused(which, bad, word):
    refused(call(which, **bad), word)


def test_nothing_to_do_is_no_error():
    none = rows8(rows=0, q=None, scale=None, scale_stride=0)
    assert call("dispatch", T=0, x=None, row_of=None, weight=None, rows=None, q=None) == B.OK
    assert call("dispatch", n_rows=0, x=None, row_of=None, weight=None, rows=None, q=none) == B.OK
    assert call("combine", T=0, rows=None, row_of=None, weight=None, add=None, y=None) == B.OK
    assert call("backward", T=0, d_y=None, rows=None, row_of=None, weight=None, d_rows=None, q=None, d_weight=None) == B.OK
    assert call("relu", rows=0, d_h=None, h_q=None, d_pre=None, q=none) == B.OK


@needs_no_gpu
def test_correct_arguments_get_as_far_as_the_missing_device():
    none = rows8(rows=0, q=None, scale=None, scale_stride=0)
    for which, kw in (("dispatch", {}), ("dispatch", dict(rows=None)), ("dispatch", dict(q=None, weight=None)), ("dispatch", dict(q=rows8(dtype=B.E4M3 | POW2))),
                      ("dispatch", dict(T=(1 << 26) - 4, copies=1, q=None)), ("combine", {}), ("combine", dict(weight=None, add=None)), ("combine", dict(n_rows=0, rows=None)), ("backward", {}),
                      ("backward", dict(d_weight=None, rows=None)), ("backward", dict(d_rows=None, q=None)), ("backward", dict(n_rows=0, rows=None, d_rows=None, q=none)), ("relu", {}),
                      ("relu", dict(d_pre=None)), ("relu", dict(q=None)), ("relu", dict(h_dtype=B.E5M2 | POW2)), ("gradient", {}), ("gradient", dict(x=rows8(dtype=B.E5M2 | POW2))),
                      ("gradient", dict(x=none, d_y=None)), ("gradient", dict(d_y_dtype=B.F16, add=None)), ("gradient", dict(d_y_dtype=B.F32, d_w_dtype=B.F16))):
        assert call(which, **kw) == B.ENODEVICE, (which, kw, B.last_error())
        assert "no HIP device" in B.last_error()


@needs_no_gpu
def test_scales_that_are_powers_of_two_are_a_type_of_rows_of_the_other_operators():
    weights = byref(B.FP8Weights(P, P, 4, 200, 300))
    assert B.lib.pgmoe_quantize_rows(P, 200, B.F32, 8, None, 1, byref(rows8(dtype=B.E4M3 | POW2)), None) == B.ENODEVICE
    assert B.lib.pgmoe_expert_matmul(byref(rows8(dtype=B.E4M3 | POW2)), weights, P, 0, None, 0, 0, byref(rows8(cols=300, q_stride=384, dtype=B.E5M2 | POW2)), None) == B.ENODEVICE
    x = byref(rows8(rows=4096, scale_stride=4096, dtype=B.E4M3 | POW2))
    for dtype in (B.E4M3, B.E5M2):
        assert B.lib.pgmoe_expert_matmul_kernel_name(x, weights, dtype | POW2) == B.lib.pgmoe_expert_matmul_kernel_name(x, weights, dtype)
    refused(B.lib.pgmoe_quantize_rows(P, 200, B.F32, 8, None, 1, byref(rows8(dtype=POW2)), None), "dtype")
    refused(B.lib.pgmoe_quantize_rows(P, 200, B.F32 | POW2, 8, None, 1, byref(rows8()), None), "x_dtype")


def test_workspace_of_the_weight_gradient():
    for args in ((0, 8, 512, 512), (64, 0, 512, 512), (64, 8, 0, 512), (64, 8, 512, -1)):
        assert B.expert_weight_gradient_workspace_bytes(*args) == 0
    assert B.expert_weight_gradient_workspace_bytes(32768, 64, 1024, 4096) == 0          # many matrices
    # one matrix and many rows, in parts: planes of float32; the sizes its rule was measured at, both sides
    for rows, E, n_in, n_out, parts in ((512, 1, 512, 1024, 1), (1024, 1, 512, 1024, 4), (4096, 1, 512, 1024, 16), (1 << 24, 1, 512, 1024, 16), (1024, 1, 1024, 4096, 1), (4096, 1, 1024, 4096, 2),
                                        (4096, 8, 512, 512, 1), (16384, 8, 512, 512, 4), (32768, 8, 1024, 1024, 1)):
        assert B.expert_weight_gradient_workspace_bytes(rows, E, n_in, n_out) == (4 * parts * E * n_in * n_out if parts > 1 else 0), (rows, E, n_in, n_out)
    assert B.expert_weight_gradient_workspace_bytes((1 << 31) - 1, 1, 1 << 22, 1 << 22) == 0


# ------------------------------------------------------------------------------------ the binding
class OnGpu(torch.Tensor):
    """A tensor that says it is on a GPU (or, set, on another): no launch follows."""
    gpu = 0

    def get_device(self):
        return self.gpu


def calls(on=lambda t: t.as_subclass(OnGpu)):
    """Every operator with tensors that fit: (name, call, tensors by name)."""
    new = lambda *s, dtype=torch.float32: on(torch.zeros(s, dtype=dtype))  # noqa: E731
    i32, f8 = torch.int32, torch.float8_e4m3fn
    return [("pgmoe_dispatch_rows", B.dispatch_rows, dict(x=new(4, 100), row_of=new(8, dtype=i32), rows=new(8, 100), q=new(8, 128, dtype=f8), scale=new(1, 8), weight=new(4, 2))),
            ("pgmoe_combine_rows", B.combine_rows, dict(rows=new(8, 100), row_of=new(4, 2, dtype=i32), y=new(4, 100), weight=new(4, 2), add=new(4, 100))),
            ("pgmoe_combine_rows_backward", B.combine_rows_backward, dict(d_y=new(4, 100), rows=new(8, 100), row_of=new(8, dtype=i32), weight=new(4, 2), d_rows=new(8, 100),
                                                                          d_weight=new(4, 2), q=new(8, 128, dtype=f8), scale=new(1, 8))),
            ("pgmoe_relu_backward", B.relu_backward, dict(d_h=new(8, 100), h_q=new(8, 128, dtype=f8), d_pre=new(8, 100), q=new(8, 128, dtype=f8), scale=new(1, 8))),
            ("pgmoe_expert_weight_gradient", B.expert_weight_gradient, dict(x_q=new(8, 128, dtype=f8), x_scale=new(1, 8), d_y=new(8, 60), expert_offsets=new(4, dtype=i32),
                                                                            d_w=new(3, 100, 60), add=new(3, 100, 60), workspace=new(16, dtype=torch.uint8)))]


@pytest.mark.parametrize("which", range(5))
def test_binding_refuses_tensors_that_are_not_on_the_current_gpu(monkeypatch, which):
    launched = []
    name, go, tensors = calls()[which]
    monkeypatch.setattr(B.lib, name, lambda *a: launched.append(a) or B.OK)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    go(**tensors, stream=0)
    assert len(launched) == 1
    for arg, t in tensors.items():
        with pytest.raises(ValueError, match="tensors on"):
            go(**dict(tensors, **{arg: torch.zeros_like(t.as_subclass(torch.Tensor))}), stream=0)      # on the CPU
    with pytest.raises(ValueError, match="GPU"):
        go(**{a: t.as_subclass(torch.Tensor) for a, t in tensors.items()}, stream=0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="cuda:1"):
        go(**tensors, stream=0)
    assert len(launched) == 1


@pytest.mark.parametrize("which", range(5))
def test_binding_launches_on_torchs_current_stream_or_the_given_one(monkeypatch, which):
    launched = []
    name, go, tensors = calls()[which]
    monkeypatch.setattr(B.lib, name, lambda *a: launched.append(a[-1]) or B.OK)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_current_stream", lambda gpu: 0x1230 + gpu)
    Other = type("Other", (), {"cuda_stream": 0x4560})
    for kw in ({}, dict(stream=Other), dict(stream=0x7890), dict(stream=0)):
        go(**tensors, **kw)
    assert [None if s is None else s.value for s in launched] == [0x1230, 0x4560, 0x7890, None]


@pytest.mark.parametrize("which,change,error", [
    (0, dict(x=torch.zeros(4, 99)), ValueError), (0, dict(row_of=torch.zeros(7, dtype=torch.int32)), ValueError), (0, dict(row_of=torch.zeros(0, dtype=torch.int32)), ValueError),
    (0, dict(row_of=torch.zeros(8)), TypeError), (0, dict(rows=None, q=None, scale=None), ValueError), (0, dict(scale=None), ValueError), (0, dict(q=None), ValueError),
    (0, dict(weight=torch.zeros(4, 3)), ValueError), (0, dict(weight=torch.zeros(4, 2).double()), TypeError), (0, dict(rows=torch.zeros(8, 100).double()), TypeError),
    (0, dict(q=torch.zeros(7, 128).to(torch.float8_e4m3fn), scale=torch.zeros(1, 7)), ValueError), (0, dict(rows=torch.zeros(100, 8).t()), ValueError),
    (1, dict(rows=torch.zeros(8, 99)), ValueError), (1, dict(add=torch.zeros(4, 100).half()), TypeError), (1, dict(add=torch.zeros(3, 100)), ValueError),
    (1, dict(row_of=torch.zeros(3, 3, dtype=torch.int32)), ValueError), (1, dict(row_of=torch.zeros(2, 4, dtype=torch.int32).t()), ValueError),
    (2, dict(d_rows=torch.zeros(8, 100).half()), TypeError), (2, dict(d_rows=torch.zeros(7, 100)), ValueError), (2, dict(d_weight=torch.zeros(8)), ValueError),
    (2, dict(rows=None, d_rows=None, q=None, scale=None), ValueError), (2, dict(rows=torch.zeros(9, 100)), ValueError),
    (3, dict(h_q=torch.zeros(8, 96).to(torch.float8_e4m3fn)), ValueError), (3, dict(h_q=torch.zeros(8, 128)), TypeError), (3, dict(d_pre=torch.zeros(8, 101)), ValueError),
    (4, dict(x_q=torch.zeros(8, 120).to(torch.float8_e4m3fn)), ValueError), (4, dict(d_y=torch.zeros(7, 60)), ValueError), (4, dict(expert_offsets=torch.zeros(3, dtype=torch.int32)), ValueError),
    (4, dict(add=torch.zeros(3, 100, 60).half()), TypeError), (4, dict(d_w=torch.zeros(3, 60, 100).transpose(1, 2)), ValueError), (4, dict(workspace=torch.zeros(4, 4).t()), ValueError),
    (4, dict(x_scale=torch.zeros(1, 7)), ValueError),
], ids=lambda v: ",".join(v) if isinstance(v, dict) else str(v))
def test_binding_refuses_tensors_that_do_not_fit(monkeypatch, which, change, error):
    name, go, tensors = calls()[which]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B.lib, name, lambda *a: pytest.fail("launched"))
    with pytest.raises(error):
        go(**dict(tensors, **{k: v if v is None else v.as_subclass(OnGpu) for k, v in change.items()}), stream=0)


@pytest.mark.parametrize("flat", [True, False])
@pytest.mark.parametrize("k", [1, 2, 8])
def test_binding_takes_a_batch_without_tokens(monkeypatch, k, flat):
    """Weights and their gradients [0, k], as a batch of that router has them; matrices that do not fit each other are refused for it too."""
    launched = []
    for name in ("pgmoe_dispatch_rows", "pgmoe_combine_rows", "pgmoe_combine_rows_backward"):       # the library's own answer: it has nothing to launch
        monkeypatch.setattr(B.lib, name, lambda *a, call=getattr(B.lib, name): launched.append(1) or call(*a))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    new = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype).as_subclass(OnGpu)  # noqa: E731
    of = new(0, dtype=torch.int32) if flat else new(0, k, dtype=torch.int32)
    x, w = new(0, 100), new(0, k)
    for rows in (new(0, 100), new(6, 100)):
        B.dispatch_rows(x, of, rows, weight=w, stream=0)
        B.dispatch_rows(x, of, rows, stream=0)
        B.combine_rows(rows, of, x, weight=w, stream=0)
        B.combine_rows_backward(x, rows, of, w, torch.zeros_like(rows), new(0, k), stream=0)
        B.combine_rows_backward(x, rows, of, None, None, new(0, k), stream=0)
    assert len(launched) == 10
    with pytest.raises(ValueError, match="d_weight"):
        B.combine_rows_backward(x, rows, of, w, None, new(0, k + 1), stream=0)
    with pytest.raises(ValueError, match="row_of"):
        B.dispatch_rows(x, new(3, dtype=torch.int32), rows, weight=w, stream=0)


# ------------------------------------------------------------------------------------ the plain forms
@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_plain_powers_of_two(kind):
    """By hand at the borders; the code of a block's largest value is in the upper half of the type's range."""
    top = O.LARGEST[kind]
    a = np.array([0.0, top, np.nextafter(np.float32(top), np.float32(1e9)), top / 2, 1.0, top * 2.0 ** -126, top * 2.0 ** -127, top * 2.0 ** -125, 3.4e38], np.float64)
    one = 2.0 ** -8 if kind == "e4m3" else 2.0 ** -15
    assert O.least_power(a, kind).tolist() == [2.0 ** -126, 1, 2, 0.5, one, 2.0 ** -126, 2.0 ** -126, 2.0 ** -125, 2.0 ** 120 if kind == "e4m3" else 2.0 ** 113]
    g = np.random.default_rng(2)
    x = (g.standard_normal((200, 128)) * np.exp(8 * g.standard_normal((200, 1)))).astype(np.float32)
    q, s = O.block_codes(x, kind, True)
    assert np.all(np.frexp(s)[0] == 0.5) and np.all(np.abs(q).max(1) > top / 2 * (1 - 2.0 ** -4)) and np.abs(q).max() <= top
    half, least = (2.0 ** -4, 2.0 ** -10) if kind == "e4m3" else (2.0 ** -3, 2.0 ** -17)
    assert np.all(np.abs(q * s[:, None].astype(np.float64) - x) <= np.maximum(half * np.abs(x), least * s[:, None]))


def test_plain_rows_by_hand():
    x = np.array([[1.0, 2.0], [3.0, 4.0]])
    row_of = np.array([2, 0, -1, 3])
    w = np.array([[1.0, 2.0], [3.0, 4.0]])
    rows = O.dispatch_rows(x, row_of, 4, w)
    assert rows[[0, 2, 3]].tolist() == [[2, 4], [1, 2], [12, 16]] and np.isnan(rows[1]).all()
    r = np.arange(8.0).reshape(4, 2)
    y, mag = O.combine_rows(r, row_of, 2, w, add=np.array([[0.0, 0], [-100, 1]]))
    assert y.tolist() == [[4 + 0, 5 + 2], [-100 + 24, 1 + 28]] and mag.tolist() == [[4, 7], [124, 29]]
    d, mag = O.combine_weight_gradient(x, r, row_of)
    assert d.tolist() == [[4 + 10, 2], [0, 18 + 28]] and np.array_equal(d, mag)
    assert O.relu_backward(np.array([1.0, np.inf, np.nan, 2.0]), np.array([0.5, 0.0, -1.0, np.nan])).tolist() == [1, 0, 0, 2]


def test_plain_gradients_are_those_of_differences():
    """loss = <y, c>, y = combine(relu(dispatch(x) . W), w): linear between the ReLU's borders, which the steps stay clear of."""
    g = np.random.default_rng(5)
    T, k, d, f, E = 5, 2, 6, 4, 3
    counts = [4, 0, 6]
    offs = np.concatenate([[0], np.cumsum(counts)])
    row_of = g.permutation(T * k)
    row_of[3] = -1
    x, W, w, c = g.standard_normal((T, d)), g.standard_normal((E, d, f)), g.standard_normal((T, k)), g.standard_normal((T, f))
    ones = np.ones((1, T * k), np.float32)

    def forward(x, W, w):
        rows = np.nan_to_num(O.dispatch_rows(x, row_of, T * k))
        h = np.concatenate([rows[offs[e]:offs[e + 1]] @ W[e] for e in range(E)])
        return rows, h, np.maximum(h, 0), O.combine_rows(np.maximum(h, 0), row_of, T, w)[0]
    rows, pre, h, _ = forward(x, W, w)
    assert np.abs(pre[pre != 0]).min() > 1e-3
    d_h = np.nan_to_num(O.dispatch_rows(c, row_of, T * k, w))
    d_w, _ = O.combine_weight_gradient(c, h, row_of)
    d_pre = O.relu_backward(d_h, h)
    d_W, _ = O.expert_weight_gradient(rows, ones, d_pre, offs)
    d_rows = np.concatenate([d_pre[offs[e]:offs[e + 1]] @ W[e].T for e in range(E)])
    d_x, _ = O.combine_rows(d_rows, row_of, T)
    eps = 1e-6
    for got, which in ((d_x, 0), (d_W, 1), (d_w, 2)):
        for i in np.ndindex(got.shape):
            step = [np.zeros_like(a) for a in (x, W, w)]
            step[which][i] = eps
            up, down = (forward(*(a + s * e for a, e in zip((x, W, w), step)))[3] for s in (1, -1))
            # piecewise linear in each: off by rounding alone, a few 2^-53 of values of order ten, over 2 eps
            assert abs(((up - down) * c).sum() / (2 * eps) - got[i]) < 1e-7
    assert not d_W[1].any()
