"""Routing from logits and experts in 8 bits, without a GPU: what the entry points refuse, that correct arguments get as far as
the missing device, and the plain 64-bit forms against hand-made values and differences."""
import ctypes
from ctypes import byref

import numpy as np
import pytest

from oracle import operators as O
from paper_2308_12066_amd import binding as B

torch = pytest.importorskip("torch")

BUF = np.zeros(1 << 16, dtype=np.uint8)
P = BUF.ctypes.data + (-BUF.ctypes.data) % 256      # aligned host memory standing in for device pointers
needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="a launch would go through")


def router(**kw):
    base = dict(n_experts=64, top_k=4, n_groups=8, topk_groups=4, score=B.SCORE_SIGMOID, renormalize=1, scale=2.5, logits_dtype=B.BF16)
    base.update(kw)
    return B.RouterConfig(**base)


def rows(**kw):
    base = dict(q=P, q_stride=256, scale=P, scale_stride=8, rows=8, cols=200, dtype=B.E4M3)
    base.update(kw)
    return B.FP8Rows(**base)


def weights(**kw):
    base = dict(q=P, scale=P, n_experts=4, n_in=200, n_out=300)
    base.update(kw)
    return B.FP8Weights(**base)


def refused(rc, word):
    assert rc == B.EINVAL, (rc, B.last_error())
    assert word in B.last_error(), B.last_error()


@pytest.mark.parametrize("bad,word", [
    (dict(n_experts=0), "n_experts"), (dict(n_experts=257), "n_experts"), (dict(n_groups=7), "n_groups"), (dict(n_groups=-1), "n_groups"),
    (dict(n_groups=32), "n_groups"), (dict(topk_groups=9), "topk_groups"), (dict(topk_groups=-1), "topk_groups"), (dict(top_k=0), "top_k"),
    (dict(top_k=33), "top_k"), (dict(score=2), "score"), (dict(renormalize=2), "renormalize"), (dict(scale=float("nan")), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(logits_dtype=B.E4M3), "logits_dtype"),
])
def test_a_bad_router_is_refused(bad, word):
    r = router(**bad)
    refused(B.lib.pgmoe_route(byref(r), P, 256, None, 4, P, P, None, None), word)
    refused(B.lib.pgmoe_route_backward(byref(r), P, 256, P, P, None, 4, P + 4096, 256, None), word)


def test_bad_arguments_of_routing_are_refused():
    r = byref(router())
    refused(B.lib.pgmoe_route(None, P, 64, None, 4, P, P, None, None), "router")
    refused(B.lib.pgmoe_route(r, P, 63, None, 4, P, P, None, None), "logits_stride")
    refused(B.lib.pgmoe_route(r, P, 64, None, -1, P, P, None, None), "T=-1")
    refused(B.lib.pgmoe_route(r, None, 64, None, 4, P, P, None, None), "logits is NULL")
    refused(B.lib.pgmoe_route(r, P + 1, 64, None, 4, P, P, None, None), "aligned")
    refused(B.lib.pgmoe_route(r, P, 64, P + 2, 4, P, P, None, None), "bias")
    refused(B.lib.pgmoe_route(r, P, 64, None, 4, None, P, None, None), "topk_idx")
    refused(B.lib.pgmoe_route(r, P, 64, None, 4, P, None, None, None), "topk_weight")
    refused(B.lib.pgmoe_route(r, P, 64, None, 4, P, P, P + 1, None), "scores_out")
    refused(B.lib.pgmoe_route_backward(r, P, 64, P, P, None, 4, P + 8192, 63, None), "stride")
    refused(B.lib.pgmoe_route_backward(r, P, 64, None, P, None, 4, P + 8192, 64, None), "topk_idx")
    refused(B.lib.pgmoe_route_backward(r, P, 64, P, None, None, 4, P + 8192, 64, None), "d_weight")
    refused(B.lib.pgmoe_route_backward(r, P, 64, P, P, None, 4, None, 64, None), "d_logits")
    refused(B.lib.pgmoe_route_backward(r, P, 64, P, P, None, 4, P + 128, 64, None), "overlaps")


@needs_no_gpu
def test_gradient_of_routing_beside_the_logits_in_one_buffer():
    """Rows of logits and of their gradient that lie between each other share nothing; with one byte of a row in common they do."""
    r = byref(router())                                                                  # rows of 64 bf16, 128 bytes
    for stride, at in ((128, 64), (128, -64), (200, 64), (200, 136), (200, -64), (128, 64 + 128), (64, 256), (64, -256)):
        a, b = P + 16384, P + 16384 + 2 * at
        assert B.lib.pgmoe_route_backward(r, a, stride, P, P, None, 4, b, stride, None) == B.ENODEVICE, (stride, at)
    for stride, d_stride, at in ((128, 128, 63), (128, 128, 65), (200, 200, 63), (200, 200, 137), (200, 200, -63), (64, 64, 255), (128, 136, 64), (128, 128, 0)):
        a, b = P + 16384, P + 16384 + 2 * at
        refused(B.lib.pgmoe_route_backward(r, a, stride, P, P, None, 4, b, d_stride, None), "overlaps")


@pytest.mark.parametrize("bad,word", [
    (dict(dtype=B.F32), "dtype"), (dict(rows=-1), "rows"), (dict(cols=0), "columns"), (dict(cols=(1 << 22) + 1), "columns"),
    (dict(q_stride=240), "q_stride"), (dict(q_stride=264), "q_stride"), (dict(scale_stride=7), "scale_stride"), (dict(q=None), "NULL"),
    (dict(scale=None), "NULL"), (dict(q=P + 8), "aligned"), (dict(scale=P + 2), "aligned"),
])
def test_bad_rows_are_refused(bad, word):
    r = rows(**bad)
    refused(B.lib.pgmoe_quantize_rows(P, 1 << 23, B.F32, 8, None, 1, byref(r), None), word)
    if "cols" not in bad:
        refused(B.lib.pgmoe_expert_matmul(byref(r), byref(weights()), P, 0, P, 300, B.BF16, None, None), word)
        refused(B.lib.pgmoe_expert_matmul(byref(rows(cols=300, q_stride=384)), byref(weights(n_in=300, n_out=200)), P, 0, None, 0, 0, byref(r), None), word)


@pytest.mark.parametrize("bad,word", [
    (dict(n_experts=0), "n_experts"), (dict(n_experts=257), "n_experts"), (dict(n_in=0), "n_in"), (dict(n_out=(1 << 22) + 1), "n_out"),
    (dict(q=None), "NULL"), (dict(scale=None), "NULL"), (dict(q=P + 4), "aligned"),
])
def test_bad_weights_are_refused(bad, word):
    w = weights(**bad)
    refused(B.lib.pgmoe_quantize_weights(P, B.F32, byref(w), None, None), word)
    refused(B.lib.pgmoe_expert_matmul(byref(rows()), byref(w), P, 0, P, 1 << 23, B.BF16, None, None), word)


def test_bad_arguments_of_quantising_and_of_products_are_refused():
    r, w = byref(rows()), byref(weights())
    L = B.lib
    refused(L.pgmoe_quantize_rows(P, 200, B.E4M3, 8, None, 1, r, None), "x_dtype")
    refused(L.pgmoe_quantize_rows(P, 200, B.F32, -1, None, 1, r, None), "T=-1")
    refused(L.pgmoe_quantize_rows(P, 200, B.F32, 8, P, 0, r, None), "copies=0")
    refused(L.pgmoe_quantize_rows(P, 200, B.F32, 8, None, 2, r, None), "row_of")
    refused(L.pgmoe_quantize_rows(P, 200, B.F32, 9, None, 1, r, None), "row_of")
    refused(L.pgmoe_quantize_rows(P, 199, B.F32, 8, None, 1, r, None), "x_stride")
    refused(L.pgmoe_quantize_rows(None, 200, B.F32, 8, None, 1, r, None), "x is NULL")
    refused(L.pgmoe_quantize_rows(P + 2, 200, B.F32, 8, None, 1, r, None), "aligned")
    big = byref(rows(rows=8, cols=1 << 22, q_stride=1 << 22))
    refused(L.pgmoe_quantize_rows(P, 1 << 22, B.F32, (1 << 31) - 1, P, 1, big, None), "launch")
    refused(L.pgmoe_quantize_weights(P, B.F32, None, None, None), "both")
    refused(L.pgmoe_quantize_weights(None, B.F32, w, None, None), "w is NULL")
    refused(L.pgmoe_quantize_weights(P, B.E5M2, w, None, None), "w_dtype")
    refused(L.pgmoe_quantize_weights(P, B.F32, w, byref(weights()), None), "transpose")
    refused(L.pgmoe_expert_matmul(byref(rows(cols=190)), w, P, 0, P, 300, B.BF16, None, None), "columns")
    refused(L.pgmoe_expert_matmul(r, w, P, 2, P, 300, B.BF16, None, None), "relu")
    refused(L.pgmoe_expert_matmul(r, w, P, 0, None, 300, B.BF16, None, None), "exactly one")
    refused(L.pgmoe_expert_matmul(r, w, P, 0, P, 300, B.BF16, byref(rows(cols=300, q_stride=384)), None), "exactly one")
    refused(L.pgmoe_expert_matmul(r, w, P, 0, P, 299, B.BF16, None, None), "y_stride")
    refused(L.pgmoe_expert_matmul(r, w, P, 0, P, 300, B.E4M3, None, None), "y_dtype")
    refused(L.pgmoe_expert_matmul(r, w, P, 0, P + 1, 300, B.BF16, None, None), "aligned")
    refused(L.pgmoe_expert_matmul(r, w, None, 0, P, 300, B.BF16, None, None), "expert_offsets")
    refused(L.pgmoe_expert_matmul(r, w, P, 0, None, 0, 0, byref(rows(cols=299, q_stride=384)), None), "y_q")
    big = byref(rows(rows=(1 << 24) + 1, scale_stride=1 << 25))
    refused(L.pgmoe_expert_matmul(big, w, P, 0, P, 300, B.BF16, None, None), "2^24")
    big = byref(rows(rows=1 << 24, scale_stride=1 << 25))
    refused(L.pgmoe_expert_matmul(big, byref(weights(n_out=1 << 22)), P, 0, P, 1 << 22, B.BF16, None, None), "launch")


@needs_no_gpu
def test_a_grid_has_less_than_2_to_the_32_threads():
    """The largest sizes one launch holds get as far as the missing device, the next are refused."""
    L, r = B.lib, byref(router())
    for T, rc in (((1 << 28) - 16, B.ENODEVICE), ((1 << 28) - 15, B.EINVAL), ((1 << 31) - 1, B.EINVAL)):
        for got in (L.pgmoe_route(r, P, 64, None, T, P, P, None, None), L.pgmoe_route_backward(r, P, 64, P, P, None, T, P + (1 << 40), 64, None)):
            assert got == rc and (rc != B.EINVAL or "launch" in B.last_error()), T
    # 8192 blocks of 128 columns, whole 128s of rows: 8 * 256 threads each
    many = byref(rows(rows=40000, cols=1 << 20, q_stride=1 << 20, scale_stride=40000))
    assert L.pgmoe_quantize_rows(P, 1 << 20, B.F32, 255 * 128, None, 1, many, None) == B.ENODEVICE
    refused(L.pgmoe_quantize_rows(P, 1 << 20, B.F32, 255 * 128 + 1, None, 1, many, None), "launch")
    # products of few rows, 512 threads for 16 rows and 128 outputs: eight rows for each of 256 experts, and rows far apart
    for n, stride in ((256, 256), (1, 1 << 23)):
        count = n * 8 if n > 1 else 65536 + 1
        pieces = (count + 15 * n) // 16
        blocks = ((1 << 23) - 1) // pieces
        x = byref(rows(rows=count, q_stride=stride, scale_stride=count))
        for nb, rc in ((blocks, B.ENODEVICE), (blocks + 1, B.EINVAL)):
            got = L.pgmoe_expert_matmul(x, byref(weights(n_experts=n, n_out=nb * 128)), P, 0, P, nb * 128, B.BF16, None, None)
            assert got == rc and (rc != B.EINVAL or "launch" in B.last_error()), (n, nb, got)


def test_matmul_kernel_name_follows_the_launch_plan():
    """The sizes its rule was measured at, both sides."""
    few, t64, t256 = "matmul_few_rows_kernel", "matmul_tiles_kernel, 64 rows", "matmul_tiles_kernel, 256 rows"
    for each, E, n_in, n_out, name in ((8, 64, 1024, 4096, few), (12, 64, 1024, 4096, t64), (64, 8, 4096, 1024, few), (256, 1, 1024, 4096, few), (512, 1, 1024, 4096, t64),
                                       (48, 8, 1024, 4096, t64), (32, 64, 1024, 4096, t64), (64, 64, 1024, 4096, t256), (512, 8, 2048, 768, t64),
                                       (1024, 8, 2048, 768, t256), (96, 8, 1024, 4096, t64), (128, 8, 1024, 4096, t256)):
        for out in (B.F32, B.BF16, B.E4M3):
            assert B.expert_matmul_kernel_name(each * E, E, n_in, n_out, out) == name, (each, E, n_in, n_out)
    assert B.expert_matmul_kernel_name(8192, 8, 1024, 4096, q_stride=1 << 23) == few and B.expert_matmul_kernel_name(8192, 8, 1024, 4096, q_stride=(1 << 23) - 16) == t256
    assert B.expert_matmul_kernel_name(1, 256, 1, 1) == few
    assert B.expert_matmul_kernel_name(0, 8, 128, 128) is None and B.expert_matmul_kernel_name(8, 0, 128, 128) is None and B.expert_matmul_kernel_name(8, 8, 0, 128) is None
    assert B.lib.pgmoe_expert_matmul_kernel_name(None, None, 0) is None


def test_nothing_to_do_is_no_error():
    r = byref(router())
    assert B.lib.pgmoe_route(r, None, 64, None, 0, None, None, None, None) == B.OK
    assert B.lib.pgmoe_route_backward(r, None, 64, None, None, None, 0, None, 64, None) == B.OK
    none = byref(rows(rows=0, q=None, scale=None, scale_stride=0))
    assert B.lib.pgmoe_quantize_rows(None, 200, B.F32, 0, None, 1, none, None) == B.OK
    assert B.lib.pgmoe_expert_matmul(none, byref(weights()), None, 0, None, 300, B.BF16, None, None) == B.OK


@needs_no_gpu
def test_correct_arguments_get_as_far_as_the_missing_device():
    r = byref(router())
    assert B.lib.pgmoe_route(r, P, 64, P, 4, P, P, P, None) == B.ENODEVICE
    assert "no HIP device" in B.last_error()
    assert B.lib.pgmoe_route_backward(r, P, 64, P, P, P, 4, P + 8192, 64, None) == B.ENODEVICE
    assert B.lib.pgmoe_quantize_rows(P, 200, B.F32, 8, None, 1, byref(rows()), None) == B.ENODEVICE
    assert B.lib.pgmoe_quantize_weights(P, B.F32, byref(weights()), byref(weights(n_in=300, n_out=200)), None) == B.ENODEVICE
    assert B.lib.pgmoe_expert_matmul(byref(rows()), byref(weights()), P, 1, P, 300, B.F32, None, None) == B.ENODEVICE


def test_group_rows_checks_as_permute_does():
    c = B.Context(B.make_config(64, 128, 8, 2, 1, 32, B.BF16, flags=B.FLAG_HOST_ONLY))
    for args, code in (((P, 33, P, P), B.EINVAL), ((None, 4, P, P), B.EINVAL), ((P, 4, None, P), B.EINVAL), ((P, 4, P, P + 2), B.EINVAL), ((P, 4, P, P), B.ENODEVICE)):
        with pytest.raises(B.PgmoeError) as ei:
            c.group_rows(*args)
        assert ei.value.code == code
    c.close()


def test_binding_refuses_tensors_that_do_not_fit():
    z = torch.zeros(4, 64)
    R = B.Router(64, 4)
    idx, wt = torch.zeros(4, 4, dtype=torch.int32), torch.zeros(4, 4)
    with pytest.raises(ValueError):
        R.route(torch.zeros(4, 63), None, idx, wt)
    with pytest.raises(ValueError):
        R.route(torch.zeros(64, 4).t(), None, idx, wt)          # rows that are not side by side
    with pytest.raises(ValueError):
        R.route(z, torch.zeros(63), idx, wt)
    with pytest.raises(TypeError):
        R.route(z, None, idx.long(), wt)
    with pytest.raises(TypeError):
        R.route(z.double(), None, idx, wt)
    with pytest.raises(ValueError):
        R.route(z, None, idx, torch.zeros(4, 8)[:, ::2])
    q, s = torch.zeros(4, 128, dtype=torch.float8_e4m3fn), torch.zeros(1, 4)
    with pytest.raises(ValueError):
        B.quantize_rows(torch.zeros(4, 200), q, s)              # two blocks
    with pytest.raises(ValueError):
        B.quantize_rows(torch.zeros(4, 100), q, torch.zeros(1, 5))
    with pytest.raises(TypeError):
        B.quantize_rows(torch.zeros(4, 100), q.view(torch.uint8), s)
    with pytest.raises(ValueError):
        B.quantize_rows(torch.zeros(4, 100), q, s, torch.zeros(7, dtype=torch.int32), 2)
    shape, sshape = B.fp8_weight_shapes(2, 100, 300)
    wq, ws = torch.zeros(shape, dtype=torch.float8_e4m3fn), torch.zeros(sshape)
    with pytest.raises(ValueError):
        B.quantize_weights(torch.zeros(3, 100, 300), wq, ws)
    with pytest.raises(ValueError):
        B.quantize_weights(torch.zeros(2, 300, 100), wq, ws)
    with pytest.raises(ValueError):
        B.expert_matmul(q, s, wq, ws, torch.zeros(2, dtype=torch.int32), 100, 300, torch.zeros(4, 300))
    with pytest.raises(ValueError):
        B.expert_matmul(q, s, wq, ws, torch.zeros(3, dtype=torch.int32), 100, 300, torch.zeros(5, 300))


def test_a_router_shared_by_threads_keeps_the_types_of_their_logits_apart(monkeypatch):
    """Another thread's call between the preparation of a call and its launch, as a switch of threads or the released lock allow."""
    r = B.Router(8, 2)
    out = lambda: (torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))  # noqa: E731
    seen = []

    def launch(cfg, *rest):
        own = len(seen)
        seen.append(None)
        if own == 0:
            r.route(torch.zeros(4, 8, dtype=torch.bfloat16), None, *out())
        seen[own] = cfg._obj.logits_dtype
        return B.OK

    monkeypatch.setattr(B.lib, "pgmoe_route", launch)
    monkeypatch.setattr(B, "_stream_for", lambda *a: None, raising=False)      # tensors on the CPU
    r.route(torch.zeros(4, 8), None, *out())
    assert seen == [B.F32, B.BF16]


class OnGpu(torch.Tensor):
    """A tensor that says it is on a GPU (or, set, on another): no launch follows."""
    gpu = 0

    def get_device(self):
        return self.gpu


def calls(on=lambda t: t.as_subclass(OnGpu)):
    """Every operator of the binding with tensors that fit: (name, call, tensors by name)."""
    new = lambda *s, dtype=torch.float32: on(torch.zeros(s, dtype=dtype))  # noqa: E731
    r, i32, f8 = B.Router(8, 2), torch.int32, torch.float8_e4m3fn
    (sf, ssf), (sb, ssb) = B.fp8_weight_shapes(2, 100, 300), B.fp8_weight_shapes(2, 300, 100)
    route = dict(logits=new(4, 8), bias=new(8), topk_idx=new(4, 2, dtype=i32), topk_weight=new(4, 2), scores_out=new(4, 8))
    back = dict(logits=new(4, 8), topk_idx=new(4, 2, dtype=i32), d_weight=new(4, 2), d_scores=new(4, 8), d_logits=new(4, 8))
    rows = dict(x=new(4, 100), q=new(8, 128, dtype=f8), scale=new(1, 8), row_of=new(8, dtype=i32))
    weights = dict(w=new(2, 100, 300), forward_q=new(*sf, dtype=f8), forward_scale=new(*ssf), backward_q=new(*sb, dtype=f8), backward_scale=new(*ssb))
    wide = dict(x_q=new(4, 128, dtype=f8), x_scale=new(1, 4), w_q=new(*sf, dtype=f8), w_scale=new(*ssf), expert_offsets=new(3, dtype=i32), y=new(4, 300))
    eight = dict(wide, y=new(4, 384, dtype=f8), y_scale=new(3, 4))
    return [("pgmoe_route", r.route, route), ("pgmoe_route_backward", r.route_backward, back), ("pgmoe_quantize_rows", lambda **k: B.quantize_rows(copies=2, **k), rows),
            ("pgmoe_quantize_weights", B.quantize_weights, weights), ("pgmoe_expert_matmul", lambda **k: B.expert_matmul(n_in=100, n_out=300, **k), wide),
            ("pgmoe_expert_matmul", lambda **k: B.expert_matmul(n_in=100, n_out=300, **k), eight)]


@pytest.mark.parametrize("which", range(6))
def test_binding_refuses_tensors_that_are_not_on_the_current_gpu(monkeypatch, which):
    launched = []
    name, call, tensors = calls()[which]
    monkeypatch.setattr(B.lib, name, lambda *a: launched.append(a) or B.OK)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    call(**tensors, stream=0)
    assert len(launched) == 1
    for arg, t in tensors.items():
        with pytest.raises(ValueError, match="tensors on"):
            call(**dict(tensors, **{arg: torch.zeros_like(t.as_subclass(torch.Tensor))}), stream=0)      # on the CPU
    with pytest.raises(ValueError, match="GPU"):
        call(**{a: t.as_subclass(torch.Tensor) for a, t in tensors.items()}, stream=0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="cuda:1"):
        call(**tensors, stream=0)
    assert len(launched) == 1


@pytest.mark.parametrize("which", range(6))
def test_binding_launches_on_torchs_current_stream_or_the_given_one(monkeypatch, which):
    """Torch operations before and after a call run on the current stream: on another one the call would race with them."""
    launched = []
    name, call, tensors = calls()[which]
    monkeypatch.setattr(B.lib, name, lambda *a: launched.append(a[-1]) or B.OK)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    monkeypatch.setattr(B, "_current_stream", lambda gpu: 0x1230 + gpu)
    call(**tensors)
    Other = type("Other", (), {"cuda_stream": 0x4560})
    call(**tensors, stream=Other)
    call(**tensors, stream=0x7890)
    call(**tensors, stream=0)
    assert [None if s is None else s.value for s in launched] == [0x1230, 0x4560, 0x7890, None]


def test_group_rows_launches_on_torchs_current_stream_or_the_given_one(monkeypatch):
    launched = []
    monkeypatch.setattr(B.lib, "pgmoe_group_rows", lambda *a: launched.append(a[-1]) or B.OK)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    current = [0x1230]
    monkeypatch.setattr(B, "_current_stream", lambda gpu: current[gpu])
    c = B.Context(B.make_config(64, 128, 8, 2, 1, 32, B.BF16, flags=B.FLAG_HOST_ONLY))
    idx, row_of, offs = (torch.zeros(n, dtype=torch.int32).as_subclass(OnGpu) for n in (8, 8, 9))
    c.group_rows(idx, 4, row_of, offs)
    current[0] = 0
    c.group_rows(idx, 4, row_of, offs)
    c.group_rows(idx, 4, row_of, offs, 0x4560)
    c.group_rows(P, 4, P, P)                                            # addresses: the null stream, as all calls of a context
    assert [None if s is None else s.value for s in launched] == [0x1230, None, 0x4560, None]
    c.close()


# ------------------------------------------------------------------------------------ the plain forms
def test_plain_codes_are_the_types_own():
    """Every finite value of both types is its own code, and values between two go to the nearer, ties to the even one."""
    for kind, dt in (("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)):
        every = torch.arange(256, dtype=torch.uint8).view(dt).double().numpy()
        fine = np.unique(every[np.isfinite(every)])
        assert np.array_equal(O.round_to(fine, kind), fine) and fine.max() == O.LARGEST[kind]
        g = np.random.default_rng(1)
        v = np.concatenate([(fine[1:] + fine[:-1]) / 2, g.uniform(fine.min(), fine.max(), 4000), g.standard_normal(4000) * 0.01])
        assert np.array_equal(O.round_to(v, kind), torch.from_numpy(v).float().to(dt).double().numpy())


def test_plain_route_by_hand():
    z = np.log(np.array([[0.1, 0.4, 0.2, 0.3], [0.25, 0.25, 0.25, 0.25]]))
    idx, w, s = O.route(z, "softmax", 2)
    assert idx.tolist() == [[1, 3], [0, 1]] and np.allclose(w, [[0.4, 0.3], [0.25, 0.25]])
    idx, w, _ = O.route(z, "softmax", 2, renormalize=True, scale=2.0)
    assert np.allclose(w, [[8 / 7, 6 / 7], [1, 1]])
    # groups {0, 1} and {2, 3}: both are worth 0.5 in both rows, the lowest stays
    idx, _, _ = O.route(z, "softmax", 2, n_groups=2, topk_groups=1)
    assert idx.tolist() == [[1, 0], [0, 1]]
    # a bias selects but does not weigh
    idx, w, _ = O.route(z, "softmax", 1, bias=np.array([1.0, 0, 0, 0]))
    assert idx.tolist() == [[0], [0]] and np.allclose(w, [[0.1], [0.25]])
    # nothing available, and too little
    idx, w, s = O.route(np.array([[-np.inf, np.nan, -np.inf, -np.inf], [-np.inf, 0.0, np.nan, -np.inf]]), "sigmoid", 2, renormalize=True)
    assert idx.tolist() == [[0, 1], [1, 0]] and w.tolist() == [[0, 0], [1, 0]] and s.tolist() == [[0, 0, 0, 0], [0, 0.5, 0, 0]]


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("every", [False, True])
def test_plain_gradient_is_that_of_differences(kind, renormalize, every):
    g = np.random.default_rng(3)
    z, dw = g.standard_normal((5, 12)), g.standard_normal((5, 3))
    ds = g.standard_normal((5, 12)) if every else None
    z[2, 4] = -np.inf
    idx, _, _ = O.route(z, kind, 3)

    def loss(z):
        s = O.scores(z, kind)
        w = np.take_along_axis(s, idx, 1)
        w = 1.7 * (w / w.sum(1, keepdims=True) if renormalize else w)
        return (w * dw).sum() + ((s * ds).sum() if every else 0.0)
    got, _ = O.route_loss_gradient(z, idx, kind, dw, ds, renormalize, 1.7)
    h = 1e-5
    for t in range(5):
        for e in range(12):
            if z[t, e] == -np.inf:
                assert got[t, e] == 0
                continue
            d = np.zeros_like(z)
            d[t, e] = h
            # a central difference: off by h^2 / 6 times a third derivative of order one, and by rounding, 2^-53 / h
            assert abs((loss(z + d) - loss(z - d)) / (2 * h) - got[t, e]) < 1e-8


def test_tile_positions_are_a_permutation_of_whole_blocks():
    p = O.tile_positions(256, 384)
    assert np.array_equal(np.sort(p.ravel()), np.arange(256 * 384))
    assert ctypes.sizeof(B.FP8Rows) == 48 and ctypes.sizeof(B.FP8Weights) == 32 and ctypes.sizeof(B.RouterConfig) == 32
