"""The norms around a block against their plain 64-bit forms (block_reference), at the sizes and inputs where they can go wrong.

Tolerances.  u = 2^-24 is half a step of fp32.  A sum over a row adds at most 8 values in a lane, 6 times pairs of lanes and up to 16
wavefronts: 30 additions and a product each, so it is within 31 u of the sum of magnitudes, a reciprocal root within 16 + 3 u of
itself and a result of the forward within 64 u of the sum of the magnitudes it is made of.  The backward multiplies two of these: 128 u.  A
sum over rows adds at most 4 + T / 512 rows in a lane, 4 slots, 8 workgroups and 20 groups on top.  A stored value is off by half a step of its type more."""
import numpy as np
import pytest
import torch

from paper_2502_16927_amd import binding as B
import block_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CODE = {"f32": B.F32, "bf16": B.BF16}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
KIND = {"rms": B.NORM_RMS, "layer": B.NORM_LAYER}
GATE = {"none": B.GATE_NONE, "channel": B.GATE_CHANNEL, "token": B.GATE_TOKEN, "full": B.GATE_FULL}


def up(t):
    return None if t is None else t.double().cpu().numpy()


class Case:
    def __init__(self, T, d, kind="rms", gate="none", parts=3, bias=False, x="bf16", y="bf16", u="bf16", eps=1e-5, alpha=1.0, seed=0, accumulate=False):
        self.T, self.d, self.kind, self.gate, self.x_type, self.y_type, self.u_type, self.eps, self.alpha = T, d, kind, gate, x, y, u, eps, alpha
        self.post, self.pre, self.accumulate = bool(parts & B.NORM_POST), bool(parts & B.NORM_PRE), accumulate
        g = torch.Generator(device=DEV).manual_seed(seed)

        def normal(shape, mean, std, dtype=torch.float32):
            return torch.empty(shape, device=DEV).normal_(mean, std, generator=g).to(dtype)

        self.x, self.dz = normal((T, d), 0.3, 1.5, TYPE[x]), normal((T, d), 0.0, 1.0, TYPE[x])
        self.y = normal((T, d), 0.1, 0.5, TYPE[y]) if self.post else None
        self.du = normal((T, d), 0.0, 1.0, TYPE[y]) if self.pre else None
        vector = lambda there, mean: normal((d,), mean, 0.3) if there else None  # noqa: E731
        self.p = dict(post_w=vector(self.post, 1.0), post_b=vector(self.post and bias, 0.0), pre_w=vector(self.pre, 1.0), pre_b=vector(self.pre and bias, 0.0))
        self.p["gate"] = {"none": lambda: None, "channel": lambda: normal((d,), 0.5, 0.3), "token": lambda: normal((T,), 0.5, 0.3),
                          "full": lambda: normal((T, d), 0.5, 0.3, TYPE[u])}[gate]()
        self.dims = B.make_norm_dims(T, d, CODE[x], CODE[y], CODE[u], KIND[kind], parts | (B.NORM_ACCUMULATE if accumulate else 0), GATE[gate], eps, alpha)
        self.params = B.make_norm_params(**self.p)
        self.p64 = {n: up(t) for n, t in self.p.items()}
        self.z = torch.full_like(self.x, float("nan")) if self.post else None
        self.u = torch.full((T, d), float("nan"), dtype=TYPE[u], device=DEV) if self.pre else None
        self.ws = B.alloc_bytes(B.norm_workspace_bytes(self.dims))
        self.ws.fill_(255)                                           # NaN as floats: what is read was written
        nan = lambda t: None if t is None else torch.full_like(t, 0.25 if accumulate else float("nan"))  # noqa: E731
        self.g = dict(dx=torch.full_like(self.x, float("nan")), dy=torch.full((T, d), float("nan"), dtype=TYPE[u], device=DEV) if self.post else None,
                      d_gate=nan(self.p["gate"]), **{"d_" + n: nan(self.p[n]) for n in ("post_w", "post_b", "pre_w", "pre_b")})

    def forward(self, stream=None):
        B.bigmac_norm_forward(self.dims, self.params, self.x, self.y, self.z, self.u, stream)

    def stored(self):
        return self.z if self.post else self.x

    def backward(self, stream=None, dz=True):
        g = self.g
        B.bigmac_norm_backward(self.dims, self.params, self.stored() if self.pre else None, self.y, self.du, self.dz if dz else None, g["dx"], g["dy"], g["d_gate"],
                               g["d_post_w"], g["d_post_b"], g["d_pre_w"], g["d_pre_b"], self.ws, stream)

    def magnitude(self, v, w, b):
        """What a normalised value is made of, in magnitudes: |v - m| with the mean's own error, times rstd w, plus b."""
        m, r = R.statistics(v, self.kind, self.eps)
        size = (np.abs(v - m) + (np.abs(v).mean(1, keepdims=True) if self.kind == "layer" else 0.0)) * r * np.abs(w)
        return size if b is None else size + np.abs(b)

    def check_forward(self):
        x, p = up(self.x), self.p64
        if self.post:
            y = up(self.y)
            want = R.block_forward(x, y, p, self.kind, self.gate, self.eps, self.alpha)
            size = np.abs(self.alpha * x) + np.abs(R.gate_values(p["gate"], self.gate, x.shape)) * self.magnitude(y, p["post_w"], p["post_b"])
            self.near("z", self.z, want, size, 64, R.HALF_STEP[self.x_type])
        if self.pre:
            z = up(self.stored())
            self.near("u", self.u, R.norm(z, p["pre_w"], p["pre_b"], self.kind, self.eps), self.magnitude(z, p["pre_w"], p["pre_b"]), 64, R.HALF_STEP[self.u_type])

    def near(self, name, got, want, size, units, half_step):
        got = up(got)
        off = np.abs(got - want)
        # (values under the smallest normal number of bf16 and fp32 are rounded in steps of 2^-133 and 2^-149)
        limit = half_step * np.abs(want) * (1 + 2.0 ** -10) + units * R.U32 * size + 2.0 ** -133
        bad = ~(off <= limit)
        assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.size} off, first at {np.argwhere(bad)[0]}: got {got[bad][0]}, want {want[bad][0]}, limit {limit[bad][0]}"

    def check_backward(self, dz=True):
        p, g = self.p64, self.g
        z, y, du, dz = up(self.stored()) if self.pre else None, up(self.y), up(self.du), up(self.dz) if dz else None
        want = R.block_backward(z, y, du, dz, p, self.kind, self.gate, self.eps, self.alpha)
        layer = 1.0 if self.kind == "layer" else 0.0
        chain = 128 + 4 + self.T / 512 + 52
        before = 0.25 if self.accumulate else 0.0

        def input_size(v, w, c):     # magnitudes behind a row's gradient
            m, r = R.statistics(v, self.kind, self.eps)
            vh, a = (np.abs(v - m) + layer * np.abs(v).mean(1, keepdims=True)) * r, np.abs(c * w)
            return r * (a + layer * a.mean(1, keepdims=True) + vh * (a * vh).mean(1, keepdims=True)), vh

        size = np.zeros((self.T, self.d)) if dz is None else np.abs(dz)
        if self.pre:
            more, zh = input_size(z, p["pre_w"], du)
            size = size + more
            self.near("d_pre_w", g["d_pre_w"], before + want["d_pre_w"], before + (np.abs(du) * zh).sum(0), chain, R.U32)
            if g["d_pre_b"] is not None:
                self.near("d_pre_b", g["d_pre_b"], before + want["d_pre_b"], before + np.abs(du).sum(0), chain, R.U32)
        self.near("dx", g["dx"], want["dx"], abs(self.alpha) * size, 128, R.HALF_STEP[self.x_type])
        if not self.post:
            return
        gate = np.abs(R.gate_values(p["gate"], self.gate, y.shape))
        # the gradient dZ carries 128 u of its size into everything behind it
        row, yh = input_size(y, p["post_w"], gate * size)
        self.near("dy", g["dy"], want["dy"], row, 256, R.HALF_STEP[self.u_type])
        self.near("d_post_w", g["d_post_w"], before + want["d_post_w"], before + (gate * size * yh).sum(0), 128 + chain, R.U32)
        if g["d_post_b"] is not None:
            self.near("d_post_b", g["d_post_b"], before + want["d_post_b"], before + (gate * size).sum(0), 128 + chain, R.U32)
        if self.gate != "none":
            full = size * self.magnitude(y, p["post_w"], p["post_b"])
            if self.gate == "channel":
                self.near("d_gate", g["d_gate"], before + want["d_gate"], before + full.sum(0), 128 + chain, R.U32)
            else:
                self.near("d_gate", g["d_gate"], want["d_gate"], full.sum(1) if self.gate == "token" else full, 256, R.HALF_STEP["f32" if self.gate == "token" else self.u_type])

    def run(self):
        self.forward()
        self.check_forward()
        self.backward()
        self.check_backward()


# one lane, part of a wavefront, its end, the first lane of the next, every number of wavefronts, the widest; one row to many per workgroup
@pytest.mark.parametrize("d", [8, 64, 504, 512, 520, 1024, 1096, 2048, 2560, 4096, 4104, 8192])
@pytest.mark.parametrize("kind,bias", [("rms", False), ("layer", True)])
def test_widths(d, kind, bias):
    for T in (1, 5, 131):
        print(f"norms, T {T}, d {d}, {kind}", flush=True)
        Case(T, d, kind, gate="channel", bias=bias, alpha=0.75, seed=d + T).run()


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("u", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
def test_types_and_gates(x, y, u, gate):
    for kind in ("rms", "layer"):
        print(f"norms, {x} {y} {u}, gate {gate}, {kind}", flush=True)
        Case(67, 328, kind, gate=gate, x=x, y=y, u=u, alpha=1.25, bias=kind == "rms").run()


@pytest.mark.parametrize("parts", [B.NORM_PRE, B.NORM_POST])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_one_side_only(parts, kind):
    for bias in (False, True):
        Case(130, 768, kind, parts=parts, gate="token" if parts == B.NORM_POST else "none", bias=bias, x="f32").run()


def test_many_rows_and_a_bias_on_one_side():
    """More rows than a turn of the persistent workgroups holds; a bias on one side only."""
    c = Case(20011, 520, "layer", gate="channel", bias=True, y="f32")
    c.p["post_b"] = c.p64["post_b"] = c.g["d_post_b"] = None
    c.params = B.make_norm_params(**c.p)
    c.run()


def test_no_gradient_along_the_stream_and_accumulation():
    c = Case(70, 640, "rms", gate="channel", bias=True, accumulate=True, x="f32")
    c.forward()
    c.backward(dz=False)
    c.check_backward(dz=False)


def test_in_place():
    a, b = Case(33, 1024, "rms", gate="token", seed=3), Case(33, 1024, "rms", gate="token", seed=3)
    a.forward()
    b.z = b.x
    b.forward()
    assert torch.equal(a.z, b.z) and torch.equal(a.u, b.u)
    a.backward()
    b.g["dx"] = b.dz
    b.backward()
    for n in a.g:
        assert (a.g[n] is None) == (b.g[n] is None) and (a.g[n] is None or torch.equal(a.g[n], b.g[n])), n


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_rows_of_zeros_of_large_values_and_of_equal_values(kind):
    c = Case(9, 512, kind, gate="channel", x="f32", y="f32", u="f32")
    c.x[1], c.y[1] = 0.0, 0.0
    c.y[3] = c.y[3] * 1e15                                  # squares that fp32 holds, just
    c.y[5] = 3.0
    c.run()


@pytest.mark.parametrize("d", [64, 1024])
def test_a_row_with_nan_stays_alone_and_no_epsilon(d):
    """A NaN or infinity in one row leaves the others' outputs as they are; with eps 0 the places of a workgroup without a row add nothing."""
    T = 6
    a, b = (Case(T, d, "rms", gate="channel", eps=0.0, seed=5) for _ in range(2))
    b.y[2, 7], b.y[4, 0] = float("nan"), float("inf")
    for c in (a, b):
        c.forward()
        c.backward()
    a.check_forward()
    a.check_backward()
    keep = [0, 1, 3, 5]
    assert torch.equal(a.z[keep], b.z[keep]) and torch.equal(a.u[keep], b.u[keep])
    assert torch.equal(a.g["dx"][keep], b.g["dx"][keep]) and torch.equal(a.g["dy"][keep], b.g["dy"][keep])
    assert torch.isnan(b.u[2]).all() and torch.isnan(b.g["dy"][2]).any()


def test_an_infinite_gate_of_the_first_row():
    """One row of a workgroup that holds four: the other places, which have no row, add nothing to the infinite sums (their 0 times infinity would be NaN)."""
    c = Case(1, 64, "rms", gate="token", bias=True)
    c.p["gate"][0] = float("inf")
    c.forward()
    c.z.copy_(c.x)                                          # (z is not finite; a finite stream for the norm behind it)
    c.backward()
    p = {**c.p64, "gate": np.ones(1)}
    want = R.block_backward(up(c.z), up(c.y), up(c.du), up(c.dz), p, c.kind, c.gate, c.eps, c.alpha)
    for n in ("d_post_w", "d_post_b"):
        assert np.array_equal(up(c.g[n]), np.sign(want[n]) * np.inf), n
    for n in ("d_pre_w", "d_pre_b"):
        assert torch.isfinite(c.g[n]).all(), n


def test_outputs_end_where_they_end():
    """Nothing behind the last row and nothing behind the last column's vector is written."""
    T, d = 3, 72
    c = Case(T, d, "rms", gate="channel")
    room = torch.full((T * d + 256,), 7.0, dtype=torch.bfloat16, device=DEV)
    c.z, c.u = room[:T * d].view(T, d), None
    tail = torch.full((T * d + 256,), 7.0, dtype=torch.bfloat16, device=DEV)
    c.u = tail[:T * d].view(T, d)
    vec = torch.full((d + 64,), 7.0, device=DEV)
    c.g["d_pre_w"] = vec[:d]
    c.run()
    assert (room[T * d:] == 7).all() and (tail[T * d:] == 7).all() and (vec[d:] == 7).all()


def test_rows_past_32_bit_offsets():
    """5 GiB of rows: the last ones, past every 32-bit byte offset, are computed like the same rows alone."""
    d, T = 8192, 327681
    x = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    x[-64:].normal_(0.0, 1.0, generator=torch.Generator(device=DEV).manual_seed(1))
    x[:-64] = 1.0
    w = torch.rand(d, device=DEV)
    p = B.make_norm_params(pre_w=w)
    u = torch.empty_like(x)
    B.bigmac_norm_forward(B.make_norm_dims(T, d, parts=B.NORM_PRE), p, x, None, None, u)
    few = torch.empty((64, d), dtype=torch.bfloat16, device=DEV)
    B.bigmac_norm_forward(B.make_norm_dims(64, d, parts=B.NORM_PRE), p, x[-64:], None, None, few)
    assert torch.equal(u[-64:], few)
    assert torch.equal(u[0], u[T - 65]) and float((u[0].double() - w.double() / (1 + 1e-5) ** 0.5).abs().max()) < 2.0 ** -8


def test_other_stream_and_equal_bits():
    a, b = (Case(3000, 640, "layer", gate="full", bias=True, seed=9) for _ in range(2))
    a.forward()
    a.backward()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    b.forward(stream=s.cuda_stream)
    b.backward(stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(a.z, b.z) and torch.equal(a.u, b.u)
    for n in a.g:
        assert a.g[n] is None or torch.equal(a.g[n], b.g[n]), n


def test_graph_replays_equal_eager():
    c = Case(700, 1024, "rms", gate="channel", bias=True, y="f32")
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    outs = {"z": c.z, "u": c.u, **{n: t for n, t in c.g.items() if t is not None}}
    want = {n: t.clone() for n, t in outs.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        c.backward()
    for replay in range(4):
        for t in outs.values():
            t.fill_(float("nan"))
        _ = (c.x.float() * 2).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in outs.items():
            assert torch.equal(t, want[n]), f"replay {replay}: {n}"


def test_branch_and_backward_past_32_bit_offsets():
    """5 GiB a tensor: the last rows, past every 32-bit byte offset, go forward through a branch and back like the same rows alone."""
    d, T, n = 8192, 327681, 64
    g = torch.Generator(device=DEV).manual_seed(2)
    w = torch.rand((2, d), generator=g, device=DEV) + 0.5
    p = B.make_norm_params(post_w=w[0], pre_w=w[1])

    def tensor(rows, fill=None):
        t = torch.empty((rows, d), dtype=torch.bfloat16, device=DEV)
        if fill is not None:
            t[:-n] = fill
            t[-n:].normal_(0.0, 1.0, generator=g)
        return t

    x, y, du, dz = tensor(T, 1.0), tensor(T, 1.0), tensor(T, 0.0), tensor(T, 0.0)

    def step(x, y, du, dz):
        rows = x.shape[0]
        dims = B.make_norm_dims(rows, d)
        z, u, dx, dy = (tensor(rows) for _ in range(4))
        vectors = torch.empty((2, d), device=DEV)
        B.bigmac_norm_forward(dims, p, x, y, z, u)
        B.bigmac_norm_backward(dims, p, z, y, du, dz, dx, dy, None, vectors[0], None, vectors[1], None, B.alloc_bytes(B.norm_workspace_bytes(dims)))
        return z, u, dx, dy, vectors

    print(f"norms of {T} rows", flush=True)
    many, few = step(x, y, du, dz), step(*(t[-n:] for t in (x, y, du, dz)))
    for name, a, b in zip(("z", "u", "dx", "dy"), many, few):
        assert torch.equal(a[-n:], b), name
    assert (many[2][:-n] == 0).all() and (many[3][:-n] == 0).all()
    # the other rows add nothing; the sums of 64 rows in two orders are within 63 roundings each of the sum of magnitudes, which the values bound
    off = (many[4].double() - few[4].double()).abs()
    z, y64, du64, dz64 = (t.double() for t in (few[0], y[-n:], du[-n:], dz[-n:]))
    unit = lambda v: v / (v.square().mean(1, keepdim=True) + 1e-5).sqrt()  # noqa: E731
    pre = du64.abs() * unit(z).abs()
    a = du64 * w[1].double()
    dZ = dz64 + (a - unit(z) * (a * unit(z)).mean(1, keepdim=True)) / (z.square().mean(1, keepdim=True) + 1e-5).sqrt()
    post = dZ.abs() * unit(y64).abs()
    limit = torch.stack([post.sum(0), pre.sum(0)]) * 2 * 70 * R.U32
    assert (off <= limit * 1.01).all()
