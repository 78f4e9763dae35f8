"""The operators around the layer as a user's program calls them: the norms before and after the block with its gate and
residual scale (forward, and backward from what the forward left), and the 4-bit path of serving - rows and weights into
microscaled 4-bit floating point and back, the product of two such operands, the experts' FFN on them.

Two forms of each: the plain one in elementary torch operations in 32 bits, and the library's calls (own = True).
Letters: T tokens, d model width, r low width, N experts, k experts per token, h expert hidden width.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _norm(name, kind, T, d, norm="rms", post=True, pre=True, gate="channel", alpha=1.0, bias=False, x="bf16", y="bf16", u="bf16"):
    case = dict(kind=kind, T=T, d=d, norm=norm, post=post, pre=pre, gate=gate, alpha=alpha, bias=bias, x=x, y=y, u=u)
    return dict(case, name=name) if name else case


def _mx(name, kind, **sizes):
    case = dict(kind=kind, **sizes)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one token being decoded, the norm in front of the block only: launches and latency
        _norm("norm_one_token", "norm_forward", 1, 4096, post=False, gate="none"),
        # a decode step of a busy server: norm behind one block, gate, residual, norm in front of the next
        _norm("norm_decode_500", "norm_forward", 500, 4096),
        # the same step of a training batch of a large layer, whose y is fp32
        _norm("norm_train_forward", "norm_forward", 32768, 4096, alpha=0.5, y="f32"),
        # backward of a mid-size GPT layer: layer norms with biases, one gate value per token, an fp32 residual stream, a ragged batch
        _norm("norm_layer_backward", "norm_backward", 6001, 1024, norm="layer", gate="token", bias=True, x="f32", y="f32"),
        # backward of the large layer
        _norm("norm_train_backward", "norm_backward", 32768, 4096, alpha=0.5, y="f32"),
        # the tokens of a prefill chunk into 4 bits and read back, a ragged count
        _mx("mx_rows_16001", "rows", rows=16001, cols=1024, dtype="bf16"),
        # an expert matrix set of the large layer laid out once at load time, and read back for a check
        _mx("mx_weights_64", "weights", N=64, n_in=1024, n_out=4096, dtype="bf16"),
        # the descending projection of a prefill chunk: one dense product
        _mx("mx_descend_2048", "product", rows=2048, N=1, n_in=4096, n_out=1024, out="bf16", bias=False, spread=0.0),
        # decode steps of the large layer's experts: every expert's weights read for four rows each ...
        _mx("mx_experts_32", "ffn", T=32, d=4096, r=1024, N=64, k=8, h=4096, bias=False, spread=0.0),
        # ... and for sixty, with biases
        _mx("mx_experts_500", "ffn", T=500, d=4096, r=1024, N=64, k=8, h=4096, bias=True, spread=0.3),
        # a prefill chunk
        _mx("mx_experts_2048", "ffn", T=2048, d=4096, r=1024, N=64, k=8, h=4096, bias=False, spread=0.3),
        # evaluation on a large batch: the matrix cores' case
        _mx("mx_experts_16384", "ffn", T=16384, d=4096, r=1024, N=64, k=8, h=4096, bias=False, spread=0.3),
    ]


_MAX_ELEMENTS = 32768 * 4096                     # of a norm's tensor
_MAX_PRODUCT = 16384 * 8 * 1024 * 4096           # rows x matrix of the experts
_MAX_WEIGHTS = 64 * 1024 * 4096


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["norm_forward", "norm_backward", "rows", "weights", "product", "ffn"], [0.22, 0.22, 0.08, 0.08, 0.14, 0.26])[0]
    if kind.startswith("norm"):
        d = 64 * _log_int(rng, 4, 64)            # 256 .. 4096
        T = _log_int(rng, 1 if kind == "norm_forward" else 64, min(32768, _MAX_ELEMENTS // d))
        post = rng.random() < 0.8
        pre = not post or rng.random() < 0.8
        gate = rng.choice(["none", "channel", "token", "full"]) if post else "none"
        return _norm(None, kind, T, d, norm=rng.choice(["rms", "rms", "layer"]), post=post, pre=pre, gate=gate, alpha=rng.choice([1.0, 0.5, 1.25]) if post else 1.0,
                     bias=rng.random() < 0.3, x=rng.choice(["bf16", "f32"]), y=rng.choice(["bf16", "f32"]), u=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "rows":
        return _mx(None, kind, rows=_log_int(rng, 1, 65536), cols=32 * _log_int(rng, 4, 128), dtype=rng.choice(["bf16", "f32"]))
    while True:
        n_in, n_out, N = 64 * _log_int(rng, 2, 64), 64 * _log_int(rng, 2, 64), rng.choice([8, 16, 48, 64, 128])
        if kind == "weights":
            if N * n_in * n_out <= _MAX_WEIGHTS:
                return _mx(None, kind, N=N, n_in=n_in, n_out=n_out, dtype=rng.choice(["bf16", "f32"]))
            continue
        if kind == "product":
            N = rng.choice([1, 1, 8, 32])
            rows = _log_int(rng, 1, 16384)
            if N * n_in * n_out <= _MAX_WEIGHTS:
                return _mx(None, kind, rows=rows, N=N, n_in=n_in, n_out=n_out, out=rng.choice(["bf16", "f32"]), bias=rng.random() < 0.3, spread=rng.choice([0.0, 0.3]))
            continue
        r = 64 * _log_int(rng, 2, 16)            # 128 .. 1024
        h = r * rng.choice([2, 4])
        k = rng.choice([1, 2, 4, 6, 8])
        T = _log_int(rng, 1, 16384)
        if T * k * r * h <= _MAX_PRODUCT and N * r * h <= _MAX_WEIGHTS:
            return _mx(None, kind, T=T, d=4 * r, r=r, N=N, k=k, h=h, bias=rng.random() < 0.3, spread=rng.choice([0.0, 0.3]))


# ------------------------------------------------------------------ inputs

def _normal(g, shape, std, dtype, mean=0.0):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(mean, std, generator=g).to(dtype)


def _offsets(rows, N, spread, seed):
    """Rows per expert as a router hands them out (spread: relative deviation of the experts' popularity)."""
    g = torch.Generator()
    g.manual_seed(seed)
    popular = (1.0 + spread * torch.randn(N, generator=g)).clamp_min(0.05)
    counts = torch.bincount(torch.multinomial(popular, rows, replacement=True, generator=g), minlength=N)
    return torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).to(torch.int32).to(DEV), int(counts.max())


def _quantised(v, dim):
    """The values that 4 bits hold of v (fp32 in, fp32 out), in blocks of 32 along dim: a block's scale is 2^(floor(log2 of its largest
    magnitude) - 2); what is left is rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code)."""
    shape = v.shape
    b = v.unflatten(dim, (-1, 32))
    dim = dim % len(shape) + 1
    top = b.abs().amax(dim, keepdim=True)
    scale = ((torch.frexp(top).exponent + 124) << 23).view(torch.float32)   # 2^(exponent - 3), by its bits
    q = b / scale
    a = q.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return (torch.copysign((torch.round(a / step) * step).clamp_max(6.0), q) * scale).reshape(shape)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": case}
    if case["kind"].startswith("norm"):
        T, d, tx, ty, tu = case["T"], case["d"], TYPES[case["x"]], TYPES[case["y"]], TYPES[case["u"]]

        def vector(mean, std):
            return _normal(g, (d,), std, torch.float32, mean)

        for p in ("post", "pre"):
            s[p + "_w"] = vector(1.0, 0.1) if case[p] else None
            s[p + "_b"] = vector(0.0, 0.1) if case[p] and case["bias"] else None
        s["gate"] = None
        if case["gate"] == "channel":
            s["gate"] = vector(0.5, 0.2)
        elif case["gate"] == "token":
            s["gate"] = torch.rand(T, generator=g, device=DEV)
        elif case["gate"] == "full":
            s["gate"] = torch.rand((T, d), generator=g, device=DEV).to(tu)
        branch = case["post"]                     # without: the norm in front of a block, on the residual stream as it is
        s["x"] = _normal(g, (T, d), 1.5, tx, 0.1)  # backward: the stream behind the branch, z
        s["y"] = _normal(g, (T, d), 0.4, ty, 0.05) if branch else None
        if case["kind"] == "norm_forward":
            s["z"] = torch.empty((T, d), dtype=tx, device=DEV) if branch else None
            s["u"] = torch.empty((T, d), dtype=tu, device=DEV) if case["pre"] else None
        else:
            s["du"] = _normal(g, (T, d), 1.0, ty) if case["pre"] else None
            s["dz"] = _normal(g, (T, d), 1.0, tx)
            s["dx"] = torch.empty((T, d), dtype=tx, device=DEV)
            s["dy"] = torch.empty((T, d), dtype=tu, device=DEV) if branch else None
            for n in ("gate", "post_w", "post_b", "pre_w", "pre_b"):
                s["d_" + n] = torch.empty_like(s[n]) if s[n] is not None else None
    elif case["kind"] in ("rows", "weights"):
        shape, std = ((case["rows"], case["cols"]), 1.0) if case["kind"] == "rows" else ((case["N"], case["n_in"], case["n_out"]), 0.02)
        s["src"] = _normal(g, shape, std, TYPES[case["dtype"]])
        s["values"] = torch.empty_like(s["src"])
    else:
        ffn = case["kind"] == "ffn"
        rows, wide, hid, N = (case["T"] * case["k"], case["r"], case["h"], case["N"]) if ffn else (case["rows"], case["n_in"], case["n_out"], case["N"])
        s["src"] = _normal(g, (rows, wide), 1.0, torch.bfloat16)
        s["offsets"], s["most"] = _offsets(rows, N, case["spread"], seed)
        # weights whose values 4 bits hold, so that both forms start from the same
        s["w1"] = _quantised(_normal(g, (N, wide, hid), 0.05, torch.float32), 1).to(torch.bfloat16)
        s["b1"] = _normal(g, (N, hid), 0.2, torch.bfloat16) if case["bias"] else None
        if ffn:
            s["w2"] = _quantised(_normal(g, (N, hid, wide), 0.02, torch.float32), 1).to(torch.bfloat16)
            s["b2"] = _normal(g, (N, wide), 0.02, torch.bfloat16) if case["bias"] else None
        s["out"] = torch.empty((rows, wide if ffn else hid), dtype=torch.bfloat16 if ffn else TYPES[case["out"]], device=DEV)
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program keeps between calls: sizes, workspaces, and the weights laid out once as they are loaded."""
    from paper_2502_16927_amd import binding as B
    c, code = s["case"], {"f32": B.F32, "bf16": B.BF16}
    if c["kind"].startswith("norm"):
        s["dims"] = B.make_norm_dims(c["T"], c["d"], code[c["x"]], code[c["y"]], code[c["u"]], kind=B.NORM_LAYER if c["norm"] == "layer" else B.NORM_RMS,
                                     parts=(B.NORM_POST if c["post"] else 0) | (B.NORM_PRE if c["pre"] else 0),
                                     gate={"none": B.GATE_NONE, "channel": B.GATE_CHANNEL, "token": B.GATE_TOKEN, "full": B.GATE_FULL}[c["gate"]],
                                     eps=EPS, alpha=c["alpha"])
        s["params"] = B.make_norm_params(s["post_w"], s["post_b"], s["pre_w"], s["pre_b"], s["gate"])
        if c["kind"] == "norm_backward":
            s["ws"] = B.alloc_bytes(B.norm_workspace_bytes(s["dims"]), DEV)
    elif c["kind"] == "rows":
        s["codes"] = torch.empty((c["rows"], c["cols"] // 2), dtype=torch.uint8, device=DEV)
        s["scales"] = torch.empty((c["rows"], B.mx_scale_bytes(c["cols"])), dtype=torch.uint8, device=DEV)
    elif c["kind"] == "weights":
        s["packed"] = B.alloc_bytes(B.mx_packed_bytes(c["N"], c["n_in"], c["n_out"]), DEV)
    else:
        for n in ("w1", "w2"):
            if n in s:
                N, n_in, n_out = s[n].shape
                s[n + "_packed"] = B.alloc_bytes(B.mx_packed_bytes(N, n_in, n_out), DEV)
                B.bigmac_mx_pack(N, n_in, n_out, B.BF16, s[n], s[n + "_packed"])
        if c["kind"] == "ffn":
            s["dims"] = B.make_dims(c["T"], c["d"], c["r"], c["N"], c["k"], c["h"])
            s["ws"] = B.alloc_bytes(B.workspace_bytes(s["dims"], B.WS_MX_GROUPED_FFN), DEV)
        else:
            s["codes"] = torch.empty((c["rows"], c["n_in"] // 2), dtype=torch.uint8, device=DEV)
            s["scales"] = torch.empty((c["rows"], B.mx_scale_bytes(c["n_in"])), dtype=torch.uint8, device=DEV)
            s["dims"] = B.make_mx_dims(c["rows"], c["N"], c["n_in"], c["n_out"], code[c["out"]])
            s["ws"] = B.alloc_bytes(B.mx_workspace_bytes(s["dims"]), DEV)


# ------------------------------------------------------------------ one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        return _run_own(s, kind)
    if kind == "norm_forward":
        return _norm_forward(s)
    if kind == "norm_backward":
        return _norm_backward(s)
    if kind == "rows":
        return _quantised(s["src"].float(), 1).to(s["src"].dtype)
    if kind == "weights":
        return _quantised(s["src"].float(), 1).to(s["src"].dtype)
    return _experts(s, kind == "ffn")


def _run_own(s, kind):
    from paper_2502_16927_amd import binding as B
    if kind == "norm_forward":
        B.bigmac_norm_forward(s["dims"], s["params"], s["x"], s["y"], s["z"], s["u"])
        return {"z": s["z"], "u": s["u"]}
    if kind == "norm_backward":
        B.bigmac_norm_backward(s["dims"], s["params"], s["x"], s["y"], s["du"], s["dz"], s["dx"], s["dy"], s["d_gate"], s["d_post_w"], s["d_post_b"],
                               s["d_pre_w"], s["d_pre_b"], s["ws"])
        return {n: s[n] for n in ("dx", "dy", "d_gate", "d_post_w", "d_post_b", "d_pre_w", "d_pre_b")}
    c = s["case"]
    if kind in ("rows", "weights"):
        dtype = B.BF16 if c["dtype"] == "bf16" else B.F32
        if kind == "rows":
            B.bigmac_mx_quantize(c["rows"], c["cols"], dtype, s["src"], s["codes"], s["scales"])
            B.bigmac_mx_dequantize(c["rows"], c["cols"], s["codes"], s["scales"], dtype, s["values"])
        else:
            B.bigmac_mx_pack(c["N"], c["n_in"], c["n_out"], dtype, s["src"], s["packed"])
            B.bigmac_mx_unpack(c["N"], c["n_in"], c["n_out"], s["packed"], dtype, s["values"])
        return s["values"]
    if kind == "product":
        B.bigmac_mx_quantize(c["rows"], c["n_in"], B.BF16, s["src"], s["codes"], s["scales"])
        B.bigmac_mx_product(s["dims"], s["codes"], s["scales"], s["offsets"] if c["N"] > 1 else None, s["w1_packed"], s["b1"], s["out"], s["ws"])
    else:
        B.bigmac_mx_grouped_ffn(s["dims"], s["src"], s["offsets"], s["w1_packed"], s["w2_packed"], s["out"], s["ws"], b1=s["b1"], b2=s["b2"])
    return s["out"]


def _normalised(v, layer):
    """v without its mean (layer norms) over its root mean square, and the reciprocal of that, row by row."""
    if layer:
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)
    return v * r, r


def _affine(v, w, b):
    v = v * w
    return v if b is None else v + b


def _gate(s):
    g = s["gate"]
    if g is None:
        return 1.0
    return g[:, None] if s["case"]["gate"] == "token" else g.float()


def _norm_forward(s):
    c, z = s["case"], None
    layer, stream = c["norm"] == "layer", s["x"].float()
    if c["post"]:
        n = _affine(_normalised(s["y"].float(), layer)[0], s["post_w"], s["post_b"])
        z = (c["alpha"] * stream + _gate(s) * n).to(s["x"].dtype)
        stream = z.float()                        # the norm behind it reads the stream as it is stored
    u = _affine(_normalised(stream, layer)[0], s["pre_w"], s["pre_b"]).to(TYPES[c["u"]]) if c["pre"] else None
    return {"z": z, "u": u}


def _norm_input_gradient(c, v, r, layer):
    """Gradient of (v - mean) * r with respect to the row, c that of the result, v the result."""
    a = c - v * (c * v).mean(1, keepdim=True)
    if layer:
        a = a - c.mean(1, keepdim=True)
    return a * r


def _norm_backward(s):
    c = s["case"]
    layer = c["norm"] == "layer"
    out = dict.fromkeys(("dx", "dy", "d_gate", "d_post_w", "d_post_b", "d_pre_w", "d_pre_b"))
    dz = s["dz"].float()
    if c["pre"]:
        v, r = _normalised(s["x"].float(), layer)
        du = s["du"].float()
        dz = dz + _norm_input_gradient(du * s["pre_w"], v, r, layer)
        out["d_pre_w"] = (du * v).sum(0)
        out["d_pre_b"] = du.sum(0) if s["pre_b"] is not None else None
    if not c["post"]:
        out["dx"] = dz.to(s["x"].dtype)
        return out
    out["dx"] = (c["alpha"] * dz).to(s["x"].dtype)
    v, r = _normalised(s["y"].float(), layer)
    if s["gate"] is not None:
        dg = dz * _affine(v, s["post_w"], s["post_b"])
        out["d_gate"] = dg.sum(0) if c["gate"] == "channel" else dg.sum(1) if c["gate"] == "token" else dg.to(s["gate"].dtype)
    dn = dz * _gate(s)
    out["d_post_w"] = (dn * v).sum(0)
    out["d_post_b"] = dn.sum(0) if s["post_b"] is not None else None
    out["dy"] = _norm_input_gradient(dn * s["post_w"], v, r, layer).to(TYPES[c["u"]])
    return out


def _experts(s, ffn):
    """Each expert's rows, padded to the longest list of them, times its matrix: one batched product."""
    rows = s["src"].shape[0]
    offsets = s["offsets"].long()
    N = offsets.numel() - 1
    place = torch.arange(rows, device=DEV)
    expert = torch.searchsorted(offsets, place, right=True) - 1
    place = place - offsets[expert]
    padded = (offsets[:N, None] + torch.arange(s["most"], device=DEV)).clamp_max(rows - 1)
    v = torch.bmm(_quantised(s["src"].float(), 1)[padded], s["w1"].float())
    if s["b1"] is not None:
        v = v + s["b1"].float()[:, None, :]
    if ffn:
        v = _quantised(0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5))), 2)
        v = torch.bmm(v, s["w2"].float())
        if s["b2"] is not None:
            v = v + s["b2"].float()[:, None, :]
    return v[expert, place].to(s["out"].dtype)


# ------------------------------------------------------------------ the definitions in 64 bits

_HELD = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _held64(v):
    """4-bit values of the rows of v (fp64 [..., n]): of the eight magnitudes the one that is nearest, at equal distance the one with the even code."""
    b = v.reshape(-1, 32)
    top = b.abs().amax(1, keepdim=True)
    power = torch.floor(torch.log2(torch.where(top > 0, top, 1.0))).long()
    scale = ((power - 2 + 1023) << 52).view(torch.float64)
    scale = torch.where(4 * scale > top, scale / 2, torch.where(8 * scale <= top, scale * 2, scale))   # a logarithm rounded across a whole number
    a = b.abs() / scale
    best, value = torch.full_like(a, math.inf), torch.zeros_like(a)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):
        off = (a - _HELD[code]).abs()
        value = torch.where(off < best, _HELD[code], value)
        best = torch.minimum(best, off)
    return (torch.sign(b) * value * scale).reshape(v.shape)


def exact(case, seed):
    s = prepare(case, seed)
    up = lambda t: None if t is None else t.double()  # noqa: E731
    if case["kind"].startswith("norm"):
        x, y, gate = up(s["x"]), up(s["y"]), up(s["gate"])
        w = {n: up(s[n]) for n in ("post_w", "post_b", "pre_w", "pre_b")}
        if gate is not None and case["gate"] == "token":
            gate = gate.reshape(-1, 1)

        def norm(v, p):
            m = v.mean(1, keepdim=True) if case["norm"] == "layer" else 0.0
            n = w[p + "_w"] * (v - m) / torch.sqrt(((v - m) ** 2).mean(1, keepdim=True) + EPS)
            return n if w[p + "_b"] is None else n + w[p + "_b"]

        if case["kind"] == "norm_forward":
            z = case["alpha"] * x + (1.0 if gate is None else gate) * norm(y, "post") if case["post"] else None
            stored = x if z is None else z.to(s["x"].dtype).double()
            return {"z": z, "u": norm(stored, "pre") if case["pre"] else None}
        # the gradients by differentiating the definitions
        leaves = [t.requires_grad_() for t in (x, y, gate, *w.values()) if t is not None]
        if case["pre"]:
            norm(x, "pre").backward(up(s["du"]))
        dz = up(s["dz"]) + (x.grad if x.grad is not None else 0.0)
        out = dict.fromkeys(("dx", "dy", "d_gate", "d_post_w", "d_post_b", "d_pre_w", "d_pre_b"))
        if case["post"]:
            stream = torch.zeros_like(x).requires_grad_()
            (case["alpha"] * stream + (1.0 if gate is None else gate) * norm(y, "post")).backward(dz)
            out["dx"], out["dy"] = stream.grad, y.grad
            out["d_gate"] = None if gate is None else gate.grad.reshape(s["gate"].shape)
        else:
            out["dx"] = dz
        del leaves
        return {**out, **{"d_" + n: t.grad if t is not None else None for n, t in w.items()}}
    if case["kind"] == "rows":
        return _held64(s["src"].double())
    if case["kind"] == "weights":
        return torch.stack([_held64(m.double().t().contiguous()).t() for m in s["src"]])
    out = torch.empty(s["out"].shape, dtype=torch.float64, device=DEV)
    ends = s["offsets"].tolist()
    for e, (a, b) in enumerate(zip(ends[:-1], ends[1:])):
        v = _held64(s["src"][a:b].double()) @ s["w1"][e].double()
        v = v if s["b1"] is None else v + s["b1"][e].double()
        if case["kind"] == "ffn":
            v = _held64(0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))) @ s["w2"][e].double()
            v = v if s["b2"] is None else v + s["b2"][e].double()
        out[a:b] = v
    return out


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["kind"].startswith("norm"):
        T, d, x, y, u = case["T"], case["d"], size[case["x"]], size[case["y"]], size[case["u"]]
        branch = 1 if case["post"] else 0
        gate = {"none": 0, "channel": 4 * d, "token": 4 * T, "full": T * d * u}[case["gate"]]
        vectors = 4 * d * (case["post"] + case["pre"]) * (2 if case["bias"] else 1)
        if case["kind"] == "norm_forward":
            return {"bytes": T * d * (x + branch * (y + x) + (u if case["pre"] else 0)) + gate + vectors, "flops": 10.0 * T * d}
        row = x + x + branch * (y + u) + (x + y if case["pre"] else 0)      # dz, dx; y, dy; z, du
        return {"bytes": T * d * row + 2 * gate + 2 * vectors, "flops": 25.0 * T * d}
    if case["kind"] in ("rows", "weights"):
        n = case["rows"] * case["cols"] if case["kind"] == "rows" else case["N"] * case["n_in"] * case["n_out"]
        return {"bytes": n * (2 * size[case["dtype"]] + 2 * 17 / 32), "flops": 4.0 * n}
    if case["kind"] == "product":
        rows, N, n_in, n_out = (case[n] for n in ("rows", "N", "n_in", "n_out"))
        reached = N * (1.0 - (1.0 - 1.0 / N) ** rows)
        return {"bytes": rows * (2 * n_in + size[case["out"]] * n_out) + reached * n_in * n_out * 17 / 32, "flops": 2.0 * rows * n_in * n_out}
    rows, N, r, h = case["T"] * case["k"], case["N"], case["r"], case["h"]
    reached = N * (1.0 - (1.0 - 1.0 / N) ** rows)
    return {"bytes": rows * 4 * r + reached * 2 * r * h * 17 / 32, "flops": 4.0 * rows * r * h}
