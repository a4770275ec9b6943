"""What the speed of the routing and 8-bit expert operators is measured on.

A case is one call a program makes that runs its mixture-of-experts blocks with experts held in
8-bit floating point, one scale for each block of 128:

  kind "route"            pgmoe_route: scores of the experts, selection, weights.
  kind "route_backward"   pgmoe_route_backward: the gradient of the logits.
  kind "quantize_rows"    pgmoe_quantize_rows: hidden states or gradients to 8 bits, dealt to the
                          rows of their experts on the way.
  kind "quantize_weights" pgmoe_quantize_weights: a block's experts to 8 bits, once, as operand
                          tiles of x.W and of dy.W^T.
  kind "matmul"           pgmoe_expert_matmul: rows grouped by expert through their experts' matrix.

Shapes are those the repository's other measurements use: hidden sizes 512 to 2048 with four times
as many intermediate features, 8 to 256 experts, one token to 32 k rows.

Layouts (pgmoe.h has them too).  Rows: codes [rows, 128 * blocks], zero past the last column;
scales [blocks, rows].  Weights: codes in tiles of 16 output features x 128 input features of one
expert, 2048 bytes each, [expert][feature tile][input block]; in a tile [half 64 of the inputs]
[16-byte piece][feature][input], padded with zeros to whole blocks of 128; scales
[expert][feature block][input block].
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
DIMS = (512, 768, 1024, 2048)
LEAST_SCALE = 2.0 ** -126


# ------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decoded token, two of 128 experts: latency of a step's smallest call
        _route("route_t1_e128_top2", 1, 128, 2),
        # prefill of 16384 tokens with balanced sigmoid routing: 8 of 256 experts in 4 of 8 groups, 16-bit logits
        _route("route_t16384_e256_top8_groups", 16384, 256, 8, score="sigmoid", bias=True, groups=8, keep=4, renorm=True, scale=2.5, dtype="bf16"),
        # router training with a balance loss on the scores, which puts a gradient on each of them
        _route("route_backward_t16384_e128_top2", 16384, 128, 2, kind="route_backward", every=True, renorm=True),
        # router training of an odd batch without such a loss, 16-bit logits
        _route("route_backward_t8191_e256_top8", 8191, 256, 8, kind="route_backward", score="sigmoid", renorm=True, scale=2.5, dtype="bf16"),
        # a serving batch, each token to the rows of its two experts
        {"name": "quantize_rows_t64_d1024_top2", "kind": "quantize_rows", "T": 64, "d": 1024, "copies": 2, "dtype": "bf16", "q": "e4m3"},
        # float32 gradients of a prefill-sized batch on their way back through the experts, an odd number of rows
        {"name": "quantize_rows_t8191_d4096_e5m2", "kind": "quantize_rows", "T": 8191, "d": 4096, "copies": 1, "dtype": "f32", "q": "e5m2"},
        # eight small float32 experts for serving only
        {"name": "quantize_weights_e8_512x2048", "kind": "quantize_weights", "E": 8, "n_in": 512, "n_out": 2048, "dtype": "f32", "both": False},
        # one matrix of each of a block's 128 experts, for the products of both directions
        {"name": "quantize_weights_e128_1024x4096_both", "kind": "quantize_weights", "E": 128, "n_in": 1024, "n_out": 4096, "dtype": "bf16", "both": True},
        # one decoded token through its two experts: the stream of two matrices
        _matmul("matmul_t1_top2", 2, 128, 1024, 4096, relu=True),
        # a serving batch of 64 tokens, two experts each, popular and unpopular ones: the second product, in float32
        _matmul("matmul_t64_top2_zipf", 128, 128, 4096, 1024, zipf=1.1, out="f32"),
        # the gradient of a prefill batch's hidden states, rows in e5m2, some 512 for each expert
        _matmul("matmul_r4099_e8_gradient", 4099, 8, 2048, 768, x="e5m2"),
        # a large prefill, two of 128 experts a token: the first product, ReLU and back to 8 bits for the second
        _matmul("matmul_r32768_e128_relu_e4m3", 32768, 128, 1024, 4096, relu=True, out="e4m3"),
    ]


def _route(name, T, E, k, kind="route", score="softmax", bias=False, groups=1, keep=1, renorm=False, scale=1.0, dtype="f32", every=False):
    """every: the scores of all experts are an output ("route") or bring a gradient ("route_backward")."""
    return {"name": name, "kind": kind, "T": T, "E": E, "k": k, "score": score, "bias": bias, "groups": groups, "keep": keep,
            "renorm": renorm, "scale": scale, "dtype": dtype, "every": every}


def _matmul(name, rows, E, n_in, n_out, zipf=0.0, x="e4m3", relu=False, out="bf16"):
    return {"name": name, "kind": "matmul", "rows": rows, "E": E, "n_in": n_in, "n_out": n_out, "zipf": zipf, "x": x, "relu": relu, "out": out}


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("route", "route_backward", "quantize_rows", "quantize_weights", "matmul", "matmul"))
    if kind in ("route", "route_backward"):
        E = rng.choice((8, 20, 60, 64, 96, 128, 160, 256))
        groups = rng.choice([1, 1] + [g for g in (2, 4, 5, 8) if E % g == 0])
        keep = rng.randint(max(1, groups // 2), groups)
        c = _route("", _log_uniform(rng, 1, 16384), E, rng.randint(1, min(8, E // groups * keep)), kind, rng.choice(("softmax", "sigmoid")), kind == "route" and rng.random() < 0.5,
                   groups, keep, rng.random() < 0.6, rng.choice((1.0, 2.5)), rng.choice(("f32", "bf16", "f16")), rng.random() < 0.3)
        if kind == "route_backward":
            c.update(groups=1, keep=1)
        del c["name"]
        return c
    if kind == "quantize_rows":
        d = rng.choice(DIMS + (4096, rng.randint(100, 1500)))
        return {"kind": kind, "T": _log_uniform(rng, 1, 8192), "d": d, "copies": rng.choice((1, 1, 2, 8)) if d <= 2048 else 1,
                "dtype": rng.choice(("f32", "bf16", "f16")), "q": rng.choice(("e4m3", "e5m2"))}
    d = rng.choice(DIMS[:3] + (rng.randint(130, 1000),))
    f = rng.choice((2 * d, 4 * d, rng.randint(200, 4000)))
    n_in, n_out = (d, f) if rng.random() < 0.5 else (f, d)
    if kind == "quantize_weights":
        return {"kind": kind, "E": rng.choice((4, 8, 16, 32)), "n_in": n_in, "n_out": n_out, "dtype": rng.choice(("f32", "bf16", "f16")), "both": rng.random() < 0.5}
    rows = _log_uniform(rng, 1, 16384)
    c = _matmul("", rows, rng.choice((1, 8, 16, 32, 64)), n_in, n_out, rng.choice((0.0, 0.8)) if rows < 2048 else 0.0, rng.choice(("e4m3", "e4m3", "e5m2")),
                rng.random() < 0.5, rng.choice(("bf16", "bf16", "f16", "f32", "e4m3")))
    del c["name"]
    return c


def work(c):
    e = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "e5m2": 1}
    if c["kind"] == "route":
        n = c["T"] * c["E"]
        return {"bytes": n * e[c["dtype"]] + 8 * c["T"] * c["k"] + (4 * n if c["every"] else 0), "flops": 8 * n}
    if c["kind"] == "route_backward":
        n = c["T"] * c["E"]
        return {"bytes": 2 * n * e[c["dtype"]] + 8 * c["T"] * c["k"] + (4 * n if c["every"] else 0), "flops": 10 * n}
    if c["kind"] == "quantize_rows":
        blocks = _blocks(c["d"])
        return {"bytes": c["T"] * (c["d"] * e[c["dtype"]] + c["copies"] * (132 * blocks + (4 if c["copies"] > 1 else 0))), "flops": 4 * c["T"] * c["d"]}
    pad = _blocks(c["n_in"]) * _blocks(c["n_out"])  # blocks of 128 x 128 of one matrix
    if c["kind"] == "quantize_weights":
        n = c["E"] * c["n_in"] * c["n_out"]
        return {"bytes": n * e[c["dtype"]] + c["E"] * pad * (16384 + 4) * (2 if c["both"] else 1), "flops": 4 * n}
    q = _popularity(c["E"], c["zipf"])
    active = float((1.0 - (1.0 - q) ** c["rows"]).sum())  # experts that get a row, on the mean
    out = c["rows"] * (c["n_out"] * e[c["out"]] if c["out"] not in LARGEST else 132 * _blocks(c["n_out"]))
    return {"bytes": c["rows"] * 132 * _blocks(c["n_in"]) + active * c["n_in"] * c["n_out"] + out, "flops": 2.0 * c["rows"] * c["n_in"] * c["n_out"]}


def _blocks(n):
    return (n + 127) // 128


def _popularity(E, s):
    q = torch.arange(1, E + 1, dtype=torch.float64) ** -s
    return q / q.sum()


# ------------------------------------------------------------------------------------ inputs
def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = {"case": c}
    if c["kind"] in ("route", "route_backward"):
        T, E, k = c["T"], c["E"], c["k"]
        # a trained router's logits: a spread of about 1.5, and experts that differ in popularity
        s["logits"] = (1.5 * normal(T, E) + 0.5 * normal(1, E)).to(DTYPES[c["dtype"]])
        if c["kind"] == "route":
            # what a balancing rule of fixed steps of 0.001 arrives at
            s["bias"] = torch.randint(-150, 151, (E,), generator=g, device="cuda").float() * 0.001 if c["bias"] else None
        else:
            s["idx"] = torch.topk(s["logits"].float() + normal(T, E) * 0.1, k, dim=1).indices.to(torch.int32)
            s["d_weight"] = normal(T, k)
            s["d_scores"] = 0.1 * normal(T, E) if c["every"] else None
    elif c["kind"] == "quantize_rows":
        T, d = c["T"], c["d"]
        # hidden states: most features near one, a few some twenty times larger
        s["x"] = (normal(T, d) * torch.exp(0.7 * normal(1, d))).to(DTYPES[c["dtype"]])
        s["row_of"] = torch.randperm(T * c["copies"], generator=g, device="cuda").to(torch.int32) if c["copies"] > 1 else None
    elif c["kind"] == "quantize_weights":
        s["w"] = torch.empty(c["E"], c["n_in"], c["n_out"], dtype=DTYPES[c["dtype"]], device="cuda")
        s["w"].normal_(0.0, 0.02, generator=g)
    else:
        R, E, kb, nb = c["rows"], c["E"], _blocks(c["n_in"]), _blocks(c["n_out"])
        p = _popularity(E, c["zipf"])[torch.randperm(E, generator=torch.Generator().manual_seed(seed))]
        counts = torch.bincount(torch.multinomial(p, R, replacement=True, generator=torch.Generator().manual_seed(seed + 1)), minlength=E)
        s["most"] = int(counts.max())  # rows of the expert that has most
        s["offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).to(torch.int32).cuda()
        live = (torch.arange(kb * 128, device="cuda") < c["n_in"])
        top = LARGEST[c["x"]]
        # codes as quantising normal values leaves them: a block's largest entry, about three sigma, is the type's largest
        s["x_q"] = (normal(R, kb * 128) * (top / 3)).clamp(-top, top).mul_(live).to(DTYPES[c["x"]])
        s["x_scale"] = torch.exp(0.3 * normal(kb, R)) * (3 / top)
        w = (normal(E, nb * 128, kb * 128) * (448.0 / 3.8)).clamp_(-448.0, 448.0).mul_(live).mul_((torch.arange(nb * 128, device="cuda") < c["n_out"])[:, None])
        s["w_q"] = w.to(torch.float8_e4m3fn).view(torch.uint8).view(E, nb * 8, 16, kb, 2, 4, 16).permute(0, 1, 3, 4, 5, 2, 6).contiguous().view(torch.float8_e4m3fn)
        s["w_scale"] = torch.exp(0.1 * normal(E, nb, kb)) * (0.02 * 3.8 / 448.0)
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
    if c["kind"] in ("route", "route_backward"):
        router = B.Router(c["E"], c["k"], score=B.SCORE_SIGMOID if c["score"] == "sigmoid" else B.SCORE_SOFTMAX, n_groups=c["groups"], topk_groups=c["keep"],
                          renormalize=c["renorm"], scale=c["scale"])
        if c["kind"] == "route":
            idx, weight = new(c["T"], c["k"], dtype=torch.int32), new(c["T"], c["k"])
            scores = new(c["T"], c["E"]) if c["every"] else None
            router.route(s["logits"], s["bias"], idx, weight, scores)
            return [idx, weight, scores]
        d_logits = torch.empty_like(s["logits"])
        router.route_backward(s["logits"], s["idx"], s["d_weight"], s["d_scores"], d_logits)
        return [d_logits]
    if c["kind"] == "quantize_rows":
        rows, blocks = c["T"] * c["copies"], _blocks(c["d"])
        q, scale = new(rows, blocks * 128, dtype=DTYPES[c["q"]]), new(blocks, rows)
        B.quantize_rows(s["x"], q, scale, s["row_of"], c["copies"])
        return [q, scale]
    kb, nb = _blocks(c["n_in"]), _blocks(c["n_out"])
    if c["kind"] == "quantize_weights":
        tiles = lambda a, b: (new(c["E"], a * 8, b, 2, 4, 16, 16, dtype=torch.float8_e4m3fn), new(c["E"], a, b))  # noqa: E731
        out = tiles(nb, kb) + (tiles(kb, nb) if c["both"] else (None, None))
        B.quantize_weights(s["w"], *out)
        return list(out)
    if c["out"] in LARGEST:
        y, scale = new(c["rows"], nb * 128, dtype=DTYPES[c["out"]]), new(nb, c["rows"])
    else:
        y, scale = new(c["rows"], c["n_out"], dtype=DTYPES[c["out"]]), None
    B.expert_matmul(s["x_q"], s["x_scale"], s["w_q"], s["w_scale"], s["offsets"], c["n_in"], c["n_out"], y, scale, relu=c["relu"])
    return [y, scale]


# ------------------------------------------------------------------------------------ the plain form
def _plain_route(s):
    c = s["case"]
    T, E, k = c["T"], c["E"], c["k"]
    z = s["logits"].double()  # selection in 64 bits: values next to each other decide an index
    if c["score"] == "softmax":
        e = torch.exp(z - z.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-z))
    v = score if s["bias"] is None else score + s["bias"].double()
    if c["groups"] > 1:
        grouped = v.view(T, c["groups"], E // c["groups"])
        value = grouped.sort(dim=2, descending=True).values[:, :, :2].sum(2)
        kept = value.sort(dim=1, descending=True, stable=True).indices[:, :c["keep"]]
        v = torch.full_like(grouped, -math.inf).scatter(1, kept[:, :, None].expand(-1, -1, grouped.shape[2]), grouped.gather(1, kept[:, :, None].expand(-1, -1, grouped.shape[2]))).view(T, E)
    idx = v.sort(dim=1, descending=True, stable=True).indices[:, :k]
    score = score.float()
    weight = score.gather(1, idx)
    if c["renorm"]:
        weight = weight / weight.sum(1, keepdim=True)
    return [idx.to(torch.int32), weight * c["scale"], score if c["every"] else None]


def _plain_route_backward(s):
    c = s["case"]
    z, idx = s["logits"].float(), s["idx"].long()
    if c["score"] == "softmax":
        e = torch.exp(z - z.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-z))
    g = s["d_weight"] * c["scale"]
    if c["renorm"]:
        chosen = score.gather(1, idx)
        total = chosen.sum(1, keepdim=True)
        g = (g - (g * chosen / total).sum(1, keepdim=True)) / total
    d = torch.zeros_like(z).scatter(1, idx, g)
    if s["d_scores"] is not None:
        d = d + s["d_scores"]
    d = score * (d - (score * d).sum(1, keepdim=True)) if c["score"] == "softmax" else score * (1 - score) * d
    return [d.to(s["logits"].dtype)]


def _plain_codes(blocks, kind):
    """Float32 blocks [.., values] -> their codes and scales [.., 1]."""
    top = LARGEST[kind]
    most = blocks.abs().amax(-1, keepdim=True)
    scale = (most / torch.full_like(most, top)).clamp(min=LEAST_SCALE)  # by a tensor: a division, where a Python number would be multiplied by its inverse
    return (blocks / scale).clamp(-top, top).to(DTYPES[kind]), scale


def _plain_quantize_rows(s):
    c = s["case"]
    T, blocks = c["T"], _blocks(c["d"])
    x = torch.nn.functional.pad(s["x"].float(), (0, blocks * 128 - c["d"])).view(T, blocks, 128)
    q, scale = _plain_codes(x, c["q"])
    q, scale = q.view(T, blocks * 128), scale.view(T, blocks)
    if s["row_of"] is not None:
        entry = torch.empty_like(s["row_of"]).scatter(0, s["row_of"].long(), torch.arange(T * c["copies"], dtype=torch.int32, device="cuda")).long()
        q, scale = q.view(torch.uint8)[entry // c["copies"]].view(DTYPES[c["q"]]), scale[entry // c["copies"]]
    return [q, scale.t().contiguous()]


def _tiles(codes):
    """Codes [E, features, inputs], whole blocks of 128 -> operand tiles."""
    E, n, k = codes.shape
    return codes.view(torch.uint8).view(E, n // 16, 16, k // 128, 2, 4, 16).permute(0, 1, 3, 4, 5, 2, 6).contiguous().view(codes.dtype)


def _plain_quantize_weights(s):
    c = s["case"]
    E, kb, nb = c["E"], _blocks(c["n_in"]), _blocks(c["n_out"])
    w = torch.nn.functional.pad(s["w"].float(), (0, nb * 128 - c["n_out"], 0, kb * 128 - c["n_in"])).view(E, kb, 128, nb, 128)
    codes, scale = _plain_codes(w.permute(0, 1, 3, 2, 4).reshape(E, kb, nb, 128 * 128), "e4m3")
    codes, scale = codes.view(torch.uint8).view(E, kb, nb, 128, 128), scale.view(E, kb, nb)
    forward = _tiles(codes.permute(0, 2, 4, 1, 3).reshape(E, nb * 128, kb * 128).view(torch.float8_e4m3fn))
    if not c["both"]:
        return [forward, scale.transpose(1, 2).contiguous(), None, None]
    backward = _tiles(codes.permute(0, 1, 3, 2, 4).reshape(E, kb * 128, nb * 128).view(torch.float8_e4m3fn))
    return [forward, scale.transpose(1, 2).contiguous(), backward, scale]


def _plain_matmul(s):
    c = s["case"]
    R, E, kb, nb = c["rows"], c["E"], _blocks(c["n_in"]), _blocks(c["n_out"])
    row = torch.arange(R, device="cuda")
    expert = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    x = (s["x_q"].float().view(R, kb, 128) * s["x_scale"].t()[:, :, None]).view(R, kb * 128)
    tiles, scale = s["w_q"], s["w_scale"]
    few = 4 * R <= E  # then each row takes a copy of its expert's matrix, else each expert a batch as long as the longest
    if few:
        tiles, scale = tiles.view(torch.uint8)[expert].view(tiles.dtype), scale[expert]
    w = tiles.float().permute(0, 1, 5, 2, 3, 4, 6).reshape(-1, nb, 128, kb, 128)
    w = (w * scale[:, :, None, :, None]).view(-1, nb * 128, kb * 128)
    if few:
        y = torch.bmm(w, x[:, :, None])[:, :, 0]
    else:
        place = row - s["offsets"].long()[expert]
        batch = torch.zeros(E, kb * 128, s["most"], device="cuda")
        batch[expert, :, place] = x
        y = torch.bmm(w, batch)[expert, :, place]
    if c["relu"]:
        y = torch.relu(y)
    if c["out"] in LARGEST:
        q, scale = _plain_codes(y.view(R, nb, 128), c["out"])
        return [q.view(R, nb * 128), scale.view(R, nb).t().contiguous()]
    return [y[:, :c["n_out"]].to(DTYPES[c["out"]]).contiguous(), None]


_PLAIN = {"route": _plain_route, "route_backward": _plain_route_backward, "quantize_rows": _plain_quantize_rows,
          "quantize_weights": _plain_quantize_weights, "matmul": _plain_matmul}


# ------------------------------------------------------------------------------------ in 64 bits
def _round_to(v, kind):
    """Float64 values within the range of an 8-bit type -> the nearest it has, ties to even."""
    digits, least = (4, -6) if kind == "e4m3" else (3, -14)
    exponent = torch.frexp(v).exponent.to(torch.float64) - 1
    step = torch.exp2(exponent.clamp(min=least) - (digits - 1))
    return torch.round(v / step) * step


def _exact_codes(v, kind, dims):
    """Float64 values -> (codes, scales): one scale, as it is stored in 32 bits, over `dims`."""
    top = LARGEST[kind]
    scale = (v.abs().amax(dims, keepdim=True) / top).float().clamp(min=LEAST_SCALE)
    return _round_to((v / scale.double()).clamp(-top, top), kind), scale


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] in ("route", "route_backward"):
        z = s["logits"].double()
        log_score = z - torch.logsumexp(z, 1, keepdim=True) if c["score"] == "softmax" else -torch.log1p(torch.exp(-z))
        score = torch.exp(log_score)
        if c["kind"] == "route":
            v = score + (0 if s["bias"] is None else s["bias"].double())
            if c["groups"] > 1:
                size = c["E"] // c["groups"]
                value = torch.stack([torch.topk(v[:, i * size:(i + 1) * size], min(2, size), dim=1).values.sum(1) for i in range(c["groups"])], 1)
                border = torch.topk(value, c["keep"], dim=1).values[:, -1:]
                v = torch.where((value >= border).repeat_interleave(size, 1), v, -math.inf)
            idx = torch.argsort(v, dim=1, descending=True, stable=True)[:, :c["k"]]
            weight = score.gather(1, idx)
            if c["renorm"]:
                weight = torch.softmax(log_score.gather(1, idx), 1)
            return [idx, c["scale"] * weight, score if c["every"] else None]
        # by automatic differentiation of the definition
        z = z.requires_grad_()
        score = torch.softmax(z, 1) if c["score"] == "softmax" else torch.sigmoid(z)
        weight = score.gather(1, s["idx"].long())
        if c["renorm"]:
            weight = weight / weight.sum(1, keepdim=True)
        loss = (c["scale"] * weight * s["d_weight"].double()).sum()
        if s["d_scores"] is not None:
            loss = loss + (score * s["d_scores"].double()).sum()
        return [torch.autograd.grad(loss, z)[0]]
    if c["kind"] == "quantize_rows":
        kb = _blocks(c["d"])
        x = torch.zeros(c["T"], kb * 128, dtype=torch.float64, device="cuda")
        x[:, :c["d"]] = s["x"]
        q, scale = _exact_codes(x.view(c["T"], kb, 128), c["q"], 2)
        q, scale = q.view(c["T"], -1), scale[:, :, 0].double()
        if s["row_of"] is not None:
            to = s["row_of"].long()
            q = torch.zeros(len(to), kb * 128, dtype=torch.float64, device="cuda").index_copy_(0, to, q.repeat_interleave(c["copies"], 0))
            scale = torch.zeros(len(to), kb, dtype=torch.float64, device="cuda").index_copy_(0, to, scale.repeat_interleave(c["copies"], 0))
        return [q, scale.t().contiguous()]
    kb, nb = _blocks(c["n_in"]), _blocks(c["n_out"])
    # where code (feature, input) sits in a matrix of `a` by `b` blocks
    def place(a, b):
        n, k = torch.arange(a * 128, device="cuda")[:, None], torch.arange(b * 128, device="cuda")[None, :]
        return (n // 16 * b + k // 128) * 2048 + k % 128 // 64 * 1024 + k % 64 // 16 * 256 + n % 16 * 16 + k % 16
    if c["kind"] == "quantize_weights":
        out = [[], [], [], []]
        for e in range(c["E"]):
            w = torch.zeros(kb * 128, nb * 128, dtype=torch.float64, device="cuda")
            w[:c["n_in"], :c["n_out"]] = s["w"][e]
            q, scale = _exact_codes(w.view(kb, 128, nb, 128), "e4m3", (1, 3))
            q, scale = q.view(kb * 128, nb * 128), scale[:, 0, :, 0].double()
            for i, (m, sc, a, b) in enumerate(((q.t(), scale.t(), nb, kb), (q, scale, kb, nb))[:2 if c["both"] else 1]):
                out[2 * i].append(torch.zeros(m.numel(), device="cuda").scatter_(0, place(a, b).reshape(-1), m.reshape(-1).float()))
                out[2 * i + 1].append(sc)
        shape = lambda a, b: (c["E"], a * 8, b, 2, 4, 16, 16)  # noqa: E731
        out = [torch.stack(o) if o else None for o in out]
        out[0] = out[0].view(shape(nb, kb))
        out[2] = out[2].view(shape(kb, nb)) if c["both"] else None
        return out
    at, bounds = place(nb, kb), s["offsets"].tolist()
    x = s["x_q"].double() * s["x_scale"].t().double().repeat_interleave(128, 1)
    y = torch.zeros(c["rows"], nb * 128, dtype=torch.float64, device="cuda")
    for e in range(c["E"]):
        lo, hi = bounds[e], bounds[e + 1]
        if hi > lo:
            w = s["w_q"][e].view(torch.uint8).reshape(-1)[at].view(torch.float8_e4m3fn).double()
            y[lo:hi] = x[lo:hi] @ (w * s["w_scale"][e].double().repeat_interleave(128, 0).repeat_interleave(128, 1)).t()
    if c["relu"]:
        y = y.clamp(min=0)
    if c["out"] in LARGEST:
        q, scale = _exact_codes(y.view(c["rows"], nb, 128), c["out"], 2)
        return [q.view(c["rows"], -1), scale[:, :, 0].double().t().contiguous()]
    return [y[:, :c["n_out"]].contiguous(), None]
