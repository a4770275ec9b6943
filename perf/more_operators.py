"""What the speed of the operators that train a block of 8-bit experts is measured on.

A case is one call a program makes around and behind the experts' products of perf/operators.py:

  kind "dispatch"         dispatch_rows: tokens to the rows of their experts, weighed or not, as values
                          and as 8-bit codes.
  kind "combine"          combine_rows: the experts' rows back to their tokens, weighed; without weights
                          the gradient of a dispatch.
  kind "combine_backward" combine_rows_backward: the gradients of the rows and of the weights.
  kind "relu_backward"    relu_backward: gradients through the ReLU whose result was kept in 8 bits.
  kind "weight_gradient"  expert_weight_gradient: the gradient of the experts' matrices from rows
                          that were kept in 8 bits.

Shapes are those the repository's other measurements use: hidden sizes 512 to 2048 with up to four
times as many intermediate features, 1 to 64 experts, one token to 32 k rows, one to eight experts a token.

Layouts (pgmoe.h has them too).  row_of [T * copies]: the row of a token's j-th copy, a permutation of the
rows.  Codes [rows, 128 * blocks], zero past the last column; scales [blocks, rows].  Where `pow2` is
set a block's scale is the least power of two, at least 2^-126, by which its largest magnitude is within the type.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}  # 0.875 * 2^9 and 0.875 * 2^16
EXPONENT = {"e4m3": 9, "e5m2": 16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, None: 0}
DIMS = (512, 768, 1024, 2048)


# ------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decoded token to the rows of its two experts: latency of a step's smallest call
        _rows("dispatch_t1_d1024_top2", "dispatch", 1, 1024, 2),
        # a prefill batch's gradients to the rows of two experts each, weighed, for both products of the way back (a router that is not trained)
        _rows("dispatch_t16384_d1024_top2_codes", "dispatch", 16384, 1024, 2, weight=True, q="e5m2"),
        # a serving batch of 64 tokens, two experts each, onto the residual stream
        _rows("combine_t64_d1024_top2_residual", "combine", 64, 1024, 2, weight=True, add=True),
        # the gradient of a dispatch to eight of many small experts: plain sums of eight rows
        _rows("combine_t16384_d2048_top8", "combine", 16384, 2048, 8),
        # an odd batch's gradients of rows and weights, the rows' also in 8 bits for the product with the transposed weights
        _rows("combine_backward_t8191_d768_top2_codes", "combine_backward", 8191, 768, 2, weight=True, q="e5m2"),
        # eight small experts a token, float32 gradients of the tokens
        _rows("combine_backward_t16384_d2048_top8", "combine_backward", 16384, 2048, 8, weight=True, x="f32"),
        # a serving batch's worth of rows in fine-tuning, float32 results of the product before
        {"name": "relu_backward_r128_f4096", "kind": "relu_backward", "rows": 128, "f": 4096, "x": "f32", "out": "bf16", "q": "e5m2", "pow2": True},
        # a large training batch's hidden gradients, to bfloat16 for the weights' gradient and to codes for the rows'
        {"name": "relu_backward_r32768_f4096", "kind": "relu_backward", "rows": 32768, "f": 4096, "x": "bf16", "out": "bf16", "q": "e5m2", "pow2": False},
        # fine-tuning on 64 rows: some experts have none
        _gradient("weight_gradient_r64_e16_512x2048", 64, 16, 512, 2048, out="bf16"),
        # an odd batch over eight experts, added to the float32 gradient of earlier batches
        _gradient("weight_gradient_r4099_e8_768x2048_add", 4099, 8, 768, 2048, add=True),
        # a batch whose experts differ in popularity, kept with scales that are no powers of two, 16-bit floating point gradients
        _gradient("weight_gradient_r8192_e16_zipf_f16", 8192, 16, 2048, 1024, zipf=0.8, y="f16", out="f32", pow2=False),
        # a large training batch, the first matrices of 64 experts
        _gradient("weight_gradient_r32768_e64_1024x4096", 32768, 64, 1024, 4096),
    ]


def _rows(name, kind, T, d, k, weight=False, add=False, x="bf16", out="bf16", q=None, pow2=False):
    """x: type of the tokens' side (result of "combine"), out: of the rows' side; q: codes of the rows too."""
    return {"name": name, "kind": kind, "T": T, "d": d, "k": k, "weight": weight, "add": add, "x": x, "out": out, "q": q, "pow2": pow2}


def _gradient(name, rows, E, n_in, n_out, zipf=0.0, x="e4m3", y="bf16", out="f32", add=False, pow2=True):
    return {"name": name, "kind": "weight_gradient", "rows": rows, "E": E, "n_in": n_in, "n_out": n_out, "zipf": zipf, "x": x, "y": y, "out": out, "add": add, "pow2": pow2}


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("dispatch", "combine", "combine_backward", "relu_backward", "weight_gradient", "weight_gradient", "weight_gradient"))
    value = rng.choice(("bf16", "bf16", "f16", "f32"))
    if kind == "weight_gradient":
        n_in = rng.choice(DIMS[:3] + (rng.randint(130, 1000),))
        n_out = rng.choice((2 * n_in, 2048, rng.randint(200, 2000)))
        if rng.random() < 0.5:
            n_in, n_out = n_out, n_in
        rows, E = _log_uniform(rng, 1, 16384), rng.choice((1, 4, 8, 16, 32, 64))
        c = _gradient("", rows, E, n_in, n_out, rng.choice((0.0, 0.8)) if E <= 16 else 0.0, rng.choice(("e4m3", "e4m3", "e5m2")), value, rng.choice(("f32", "f32", "bf16", "f16")),
                      rng.random() < 0.3, rng.random() < 0.7)
    elif kind == "relu_backward":
        c = {"name": "", "kind": kind, "rows": _log_uniform(rng, 1, 16384), "f": rng.choice((2048, 4096, rng.randint(100, 4000))), "x": value, "out": rng.choice(("bf16", "f16", "f32", None)),
             "q": rng.choice(("e4m3", "e5m2")), "pow2": rng.random() < 0.5}
    else:
        d, k = rng.choice(DIMS + (rng.randint(100, 1500),)), rng.choice((1, 2, 2, 3, 4, 8))
        q = rng.choice((None, "e4m3", "e5m2")) if kind != "combine" else None
        c = _rows("", kind, _log_uniform(rng, 1, 16384 * 2 // max(2, k)), d, k, kind == "combine_backward" or rng.random() < 0.5, kind == "combine" and rng.random() < 0.5, value,
                  rng.choice(("bf16", "f16", "f32")) if q is None or rng.random() < 0.7 else None, q, rng.random() < 0.5)
        if kind == "combine_backward":
            c["out"] = c["out"] or "bf16"  # the type of the rows, whose products with the gradients are the weights'
    del c["name"]
    return c


def work(c):
    codes = lambda rows, n: rows * 132 * _blocks(n) if c["q"] else 0  # noqa: E731
    if c["kind"] == "weight_gradient":
        matrices = c["E"] * c["n_in"] * c["n_out"] * BYTES[c["out"]]
        return {"bytes": c["rows"] * (132 * _blocks(c["n_in"]) + c["n_out"] * BYTES[c["y"]]) + matrices * (2 if c["add"] else 1), "flops": 2.0 * c["rows"] * c["n_in"] * c["n_out"]}
    if c["kind"] == "relu_backward":
        n = c["rows"] * c["f"]
        return {"bytes": n * (BYTES[c["x"]] + 1 + BYTES[c["out"]]) + codes(c["rows"], c["f"]), "flops": n}
    R, tokens = c["T"] * c["k"], c["T"] * c["d"] * BYTES[c["x"]]
    rows, each = R * c["d"] * BYTES[c["out"]], 4 * R * (2 if c["weight"] else 1)
    if c["kind"] == "dispatch":
        return {"bytes": tokens + rows + codes(R, c["d"]) + each, "flops": R * c["d"]}
    if c["kind"] == "combine":
        return {"bytes": tokens * (2 if c["add"] else 1) + rows + each, "flops": 2 * R * c["d"]}
    return {"bytes": tokens + 2 * rows + codes(R, c["d"]) + each + 4 * R, "flops": 3 * R * c["d"]}


def _blocks(n):
    return (n + 127) // 128


# ------------------------------------------------------------------------------------ inputs
def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = {"case": c}
    if c["kind"] == "weight_gradient":
        R, E, kb = c["rows"], c["E"], _blocks(c["n_in"])
        p = torch.arange(1, E + 1, dtype=torch.float64) ** -c["zipf"]
        counts = torch.bincount(torch.multinomial(p, R, replacement=True, generator=torch.Generator().manual_seed(seed)), minlength=E)
        counts = counts[torch.randperm(E, generator=torch.Generator().manual_seed(seed + 1))]
        s["most"] = int(counts.max())  # rows of the expert that has most
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).to(torch.int32).cuda()
        # rows as quantising hidden states leaves them: a block's largest entry, about three sigma, is near the type's largest
        live, top = torch.arange(kb * 128, device="cuda") < c["n_in"], LARGEST[c["x"]]
        s["x_q"] = (normal(R, kb * 128) * (top / 4)).clamp(-top, top).mul_(live).to(DTYPES[c["x"]])
        s["x_scale"] = torch.exp(0.5 * normal(kb, R)) * (4 / top)
        if c["pow2"]:
            s["x_scale"] = torch.exp2(torch.round(torch.log2(s["x_scale"])))
        s["d_y"] = (normal(R, c["n_out"]) * torch.exp(0.5 * normal(R, 1)) * 0.01).to(DTYPES[c["y"]])
        s["add"] = (0.1 * normal(E, c["n_in"], c["n_out"])).to(DTYPES[c["out"]]) if c["add"] else None
    elif c["kind"] == "relu_backward":
        R, f = c["rows"], c["f"]
        s["d_h"] = (0.01 * normal(R, f) * torch.exp(0.5 * normal(R, 1))).to(DTYPES[c["x"]])
        # codes of a ReLU's results: half of them zero, padded to whole blocks
        s["h_q"] = torch.zeros(R, _blocks(f) * 128, dtype=DTYPES["e4m3"], device="cuda")
        s["h_q"].view(torch.uint8)[:, :f] = (normal(R, f) * 128).clamp(0, 448).to(DTYPES["e4m3"]).view(torch.uint8)
    else:
        T, d, k = c["T"], c["d"], c["k"]
        s["row_of"] = torch.randperm(T * k, generator=g, device="cuda").to(torch.int32)
        weight = torch.exp(normal(T, k))
        s["weight"] = weight / weight.sum(1, keepdim=True) if c["weight"] else None
        if c["kind"] != "combine":  # hidden states or their gradients: a few features some times larger than most
            s["x"] = (normal(T, d) * torch.exp(0.7 * normal(1, d))).to(DTYPES[c["x"]])
        if c["kind"] != "dispatch":
            s["rows"] = normal(T * k, d).to(DTYPES[c["out"]])
        s["add"] = normal(T, d).to(DTYPES[c["x"]]) if c["add"] else None
    return s


# ------------------------------------------------------------------------------------ one pass
def run(s):
    if own:
        return _own(s)
    return _PLAIN[s["case"]["kind"]](s)


def _own(s):
    from paper_2308_12066_amd import binding as B
    c = s["case"]
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if c["kind"] == "weight_gradient":
        R, E, n_in, n_out = c["rows"], c["E"], c["n_in"], c["n_out"]
        d_w = new(E, n_in, n_out, dtype=DTYPES[c["out"]])
        need = B.expert_weight_gradient_workspace_bytes(R, E, n_in, n_out)
        B.expert_weight_gradient(s["x_q"], s["x_scale"], s["d_y"], s["offsets"], d_w, add=s["add"], pow2=c["pow2"], workspace=new(need, dtype=torch.uint8) if need else None)
        return [d_w]
    R, n = (c["rows"], c["f"]) if c["kind"] == "relu_backward" else (c["T"] * c["k"], c["d"])
    if c["kind"] == "combine":
        y = new(c["T"], n, dtype=DTYPES[c["x"]])
        B.combine_rows(s["rows"], s["row_of"], y, weight=s["weight"], add=s["add"])
        return [y]
    out = new(R, n, dtype=DTYPES[c["out"]]) if c["out"] else None
    q, scale = (new(R, _blocks(n) * 128, dtype=DTYPES[c["q"]]), new(_blocks(n), R)) if c["q"] else (None, None)
    if c["kind"] == "relu_backward":
        B.relu_backward(s["d_h"], s["h_q"], out, q, scale, pow2=c["pow2"])
        return [out, q, scale]
    if c["kind"] == "dispatch":
        B.dispatch_rows(s["x"], s["row_of"], out, q, scale, weight=s["weight"], pow2=c["pow2"])
        return [out, q, scale]
    d_weight = new(c["T"], c["k"])
    B.combine_rows_backward(s["x"], s["rows"], s["row_of"], s["weight"], out, d_weight, q, scale, pow2=c["pow2"])
    return [out, q, scale, d_weight]


# ------------------------------------------------------------------------------------ the plain form
def _plain_codes(v, c):
    """Float32 rows -> codes and scales, or nothing where the case has none."""
    if not c["q"]:
        return None, None
    R, n = v.shape
    top = LARGEST[c["q"]]
    v = torch.nn.functional.pad(v, (0, _blocks(n) * 128 - n)).view(R, _blocks(n), 128)
    most = v.abs().amax(2, keepdim=True)
    if c["pow2"]:
        part, exponent = torch.frexp(most)  # part in [1/2, 1)
        scale = torch.where(most > 0, torch.ldexp(torch.ones_like(most), (exponent - EXPONENT[c["q"]] + (part > 0.875)).clamp(min=-126)), 2.0 ** -126)
    else:
        scale = (most / torch.full_like(most, top)).clamp(min=2.0 ** -126)  # by a tensor: a division, where a Python number would be multiplied by its inverse
    q = (v / scale).clamp(-top, top).to(DTYPES[c["q"]])
    return q.view(R, -1), scale.view(R, -1).t().contiguous()


def _plain_rows(s, v):
    """Values [T, d] -> those of the rows [R, d], weighed."""
    c = s["case"]
    entry = torch.empty_like(s["row_of"]).scatter(0, s["row_of"].long(), torch.arange(c["T"] * c["k"], dtype=torch.int32, device="cuda")).long()
    v = v[entry // c["k"]]
    return v if s["weight"] is None else v * s["weight"].view(-1)[entry][:, None]


def _plain_dispatch(s):
    c = s["case"]
    v = _plain_rows(s, s["x"].float())
    return [v.to(DTYPES[c["out"]]) if c["out"] else None, *_plain_codes(v, c)]


def _plain_combine(s):
    c = s["case"]
    v = s["rows"].float()[s["row_of"].long()].view(c["T"], c["k"], c["d"])
    if s["weight"] is not None:
        v = v * s["weight"][:, :, None]
    y = v.sum(1)
    if s["add"] is not None:
        y = y + s["add"].float()
    return [y.to(DTYPES[c["x"]])]


def _plain_combine_backward(s):
    c = s["case"]
    v = _plain_rows(s, s["x"].float())
    d_weight = (s["rows"].float()[s["row_of"].long()].view(c["T"], c["k"], c["d"]) * s["x"].float()[:, None]).sum(2)
    return [v.to(DTYPES[c["out"]]), *_plain_codes(v, c), d_weight]


def _plain_relu_backward(s):
    c = s["case"]
    v = torch.where(s["h_q"][:, :c["f"]].float() <= 0, 0.0, s["d_h"].float())
    return [v.to(DTYPES[c["out"]]) if c["out"] else None, *_plain_codes(v, c)]


def _plain_weight_gradient(s):
    c = s["case"]
    R, E, kb = c["rows"], c["E"], _blocks(c["n_in"])
    row = torch.arange(R, device="cuda")
    expert = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    place = row - s["offsets"].long()[expert]
    x = (s["x_q"].float().view(R, kb, 128) * s["x_scale"].t()[:, :, None]).view(R, kb * 128)[:, :c["n_in"]]
    # each expert a batch as long as the longest
    left, right = torch.zeros(E, c["n_in"], s["most"], device="cuda"), torch.zeros(E, s["most"], c["n_out"], device="cuda")
    left[expert, :, place] = x
    right[expert, place] = s["d_y"].float()
    d_w = torch.bmm(left, right)
    if s["add"] is not None:
        d_w = d_w + s["add"].float()
    return [d_w.to(DTYPES[c["out"]])]


_PLAIN = {"dispatch": _plain_dispatch, "combine": _plain_combine, "combine_backward": _plain_combine_backward, "relu_backward": _plain_relu_backward,
          "weight_gradient": _plain_weight_gradient}


# ------------------------------------------------------------------------------------ in 64 bits
def _exact_codes(v, c):
    """Float64 rows -> (codes, scales): of the values in 32 bits, by quotients in 32 bits, as a code is defined."""
    if not c["q"]:
        return None, None
    R, n = v.shape
    nb, top = _blocks(n), LARGEST[c["q"]]
    blocks = torch.zeros(R, nb * 128, dtype=torch.float64, device="cuda")
    blocks[:, :n] = v.float().double()
    blocks = blocks.view(R, nb, 128)
    scale = torch.linalg.vector_norm(blocks, math.inf, dim=2, keepdim=True) / top
    if c["pow2"]:
        scale = torch.exp2(torch.ceil(torch.log2(scale.clamp(min=2.0 ** -126))))
        scale = torch.where(blocks.abs().amax(2, keepdim=True) <= scale / 2 * top, scale / 2, scale).clamp(min=2.0 ** -126)  # should a logarithm have come out above a whole number
    scale = scale.float().clamp(min=2.0 ** -126).double()
    digits, least = (4, -6) if c["q"] == "e4m3" else (3, -14)
    v = (blocks / scale).float().double().clamp(-top, top)
    step = torch.exp2((torch.frexp(v).exponent.to(torch.float64) - 1).clamp(min=least) - (digits - 1))
    return (torch.round(v / step) * step).view(R, -1), scale.view(R, nb).t().contiguous()


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "relu_backward":
        v = s["d_h"].double() * (s["h_q"].double()[:, :c["f"]] > 0)
        return [v if c["out"] else None, *_exact_codes(v, c)]
    if c["kind"] == "weight_gradient":
        bounds = s["offsets"].tolist()
        x = s["x_q"].double()[:, :c["n_in"]] * s["x_scale"].double().repeat_interleave(128, 0)[:c["n_in"]].t()
        d_w = torch.zeros(c["E"], c["n_in"], c["n_out"], dtype=torch.float64, device="cuda") if s["add"] is None else s["add"].double()
        for e in range(c["E"]):
            lo, hi = bounds[e], bounds[e + 1]
            if hi > lo:
                d_w[e] += x[lo:hi].t() @ s["d_y"][lo:hi].double()
        return [d_w]
    T, k, d = c["T"], c["k"], c["d"]
    at = s["row_of"].long()
    weight = torch.ones(T, k, dtype=torch.float64, device="cuda") if s["weight"] is None else s["weight"].double()
    if c["kind"] == "combine":
        y = torch.zeros(T, d, dtype=torch.float64, device="cuda") if s["add"] is None else s["add"].double()
        for j in range(k):
            y += weight[:, j:j + 1] * s["rows"][at[j::k]].double()
        return [y]
    rows, d_weight = torch.empty(T * k, d, dtype=torch.float64, device="cuda"), torch.empty(T, k, dtype=torch.float64, device="cuda")
    for j in range(k):
        rows[at[j::k]] = weight[:, j:j + 1] * s["x"].double()
        if c["kind"] == "combine_backward":
            d_weight[:, j] = torch.linalg.vecdot(s["rows"][at[j::k]].double(), s["x"].double())
    got = [rows if c["out"] else None, *_exact_codes(rows, c)]
    return got + [d_weight] if c["kind"] == "combine_backward" else got
