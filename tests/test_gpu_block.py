"""The operators around the layer together with the layer, as a transformer block uses them: a training step (norm, layer, norm with gate and
residual; their gradients in turn) and a serving step (norm, router, 4-bit projections and experts, norm), eager and captured.

Every stage is held against its plain 64-bit form on the inputs that it had (see block_reference and the tests of each operator for the
tolerances; the layer's bar is the one of the other tests, 2e-2 of the RMS), and the training step's input gradient against the
whole chain."""
import numpy as np
import pytest
import torch

from paper_2502_16927_amd import binding as B
from paper_2502_16927_amd import synth
import block_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = 2e-2


def up(t):
    return t.double().cpu().numpy()


def rms_off(got, want):
    return float(np.abs(got - want).max() / np.sqrt(np.mean(want ** 2)))


def replays_equal_eager(step, outs):
    step()
    torch.cuda.synchronize()
    want = {n: t.clone() for n, t in outs.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(3):
        for t in outs.values():
            t.fill_(0 if t.dtype == torch.uint8 else 3)
        _ = torch.ones(1000, device=DEV).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in outs.items():
            assert torch.equal(t, want[n]), f"replay {replay}: {n}"


def test_training_step(oracle):
    T, d, eps, alpha = 640, 256, 1e-5, 0.8
    wl = synth.small(T=T, d=d, r=64, N=16, k=4, h=256)
    data = synth.generate(wl)
    rng = np.random.default_rng(3)
    dims = B.dims_of(wl)
    t = {n: B.to_device(data[n], B.BF16) for n in ("w_down", "w_up", "w1", "w2")}
    wg = B.to_device(data["w_gate"], B.F32)
    params = B.make_params(t["w_down"], t["w_up"], wg, None, t["w1"], t["w2"])
    f32 = lambda *s, std=1.0, mean=0.0: torch.from_numpy((mean + std * rng.standard_normal(s)).astype(np.float32)).to(DEV)  # noqa: E731
    x, dz = f32(T, d, std=1.5), f32(T, d)
    pre_w, post_w, gate = f32(d, std=0.2, mean=1.0), f32(d, std=0.2, mean=1.0), f32(d, std=0.3, mean=0.5)
    # the stream in fp32, the layer's results in fp32, what the layer reads in bf16
    pre = B.make_norm_dims(T, d, B.F32, B.F32, B.BF16, parts=B.NORM_PRE, eps=eps)
    post = B.make_norm_dims(T, d, B.F32, B.F32, B.BF16, parts=B.NORM_POST, gate=B.GATE_CHANNEL, eps=eps, alpha=alpha)
    pre_p, post_p = B.make_norm_params(pre_w=pre_w), B.make_norm_params(post_w=post_w, gate=gate)
    empty = lambda dtype: torch.empty((T, d), dtype=dtype, device=DEV)  # noqa: E731
    o = dict(u=empty(torch.bfloat16), y=empty(torch.float32), z=empty(torch.float32), dx_post=empty(torch.float32), dy=empty(torch.bfloat16), du=empty(torch.float32),
             dx=empty(torch.float32), d_gate=torch.empty_like(gate), d_post_w=torch.empty_like(post_w), d_pre_w=torch.empty_like(pre_w))
    g = {n: torch.empty(s, device=DEV) for n, s in {"d_w_down": (d, 64), "d_w_up": (64, d), "d_w_gate": (d, 16), "d_w1": (16, 64, 256), "d_w2": (16, 256, 64)}.items()}
    saved, ws = B.alloc_bytes(B.workspace_bytes(dims, B.WS_SAVED)), B.alloc_bytes(B.workspace_bytes(dims, B.WS_LAYER_TRAIN))
    ws_pre, ws_post = B.alloc_bytes(B.norm_workspace_bytes(pre)), B.alloc_bytes(B.norm_workspace_bytes(post))

    def step():
        B.bigmac_norm_forward(pre, pre_p, x, None, None, o["u"])
        B.bigmac_layer_forward(dims, params, o["u"], o["y"], saved, ws)
        B.bigmac_norm_forward(post, post_p, x, o["y"], o["z"], None)
        B.bigmac_norm_backward(post, post_p, None, o["y"], None, dz, o["dx_post"], o["dy"], o["d_gate"], o["d_post_w"], None, None, None, ws_post)
        B.bigmac_layer_backward(dims, params, o["u"], o["dy"], saved, o["du"], g["d_w_down"], g["d_w_up"], g["d_w_gate"], g["d_w1"], g["d_w2"], ws)
        B.bigmac_norm_backward(pre, pre_p, x, None, o["du"], o["dx_post"], o["dx"], None, None, None, None, o["d_pre_w"], None, ws_pre)

    replays_equal_eager(step, {**o, **g})
    a = {n: up(v) for n, v in o.items()}
    x64, p_post = up(x), dict(post_w=up(post_w), post_b=None, gate=up(gate))
    u_want = R.norm(x64, up(pre_w), None, "rms", eps)
    assert (np.abs(a["u"] - u_want) <= R.HALF_STEP["bf16"] * 1.001 * np.abs(u_want) + 1e-5).all()
    w = [data[n] for n in ("w_gate",)] + [None] + [data[n] for n in ("w_down", "w_up", "w1", "w2")]
    u32 = a["u"].astype(np.float32)
    y_want = oracle.bigmac_forward(u32, *w, wl.k)
    assert rms_off(a["y"], y_want) < TOL
    assert rms_off(a["z"], R.block_forward(x64, a["y"], p_post, "rms", "channel", eps, alpha)) < 1e-5
    back = R.block_backward(None, a["y"], None, up(dz), p_post, "rms", "channel", eps, alpha)
    for n in ("d_gate", "d_post_w"):
        assert rms_off(a[n], back[n]) < 1e-4
    # stored in bf16: off by half a step, 2^-8 of the value, on top of the fp32 arithmetic's 1e-5 (a value of 5.3 RMS alone may be off by 0.0207 RMS)
    assert (np.abs(a["dy"] - back["dy"]) <= R.HALF_STEP["bf16"] * 1.001 * np.abs(back["dy"]) + 1e-5 * np.sqrt(np.mean(back["dy"] ** 2))).all()
    grads = oracle.bigmac_backward(u32, a["dy"].astype(np.float32), *w, wl.k)
    assert rms_off(a["du"], grads["dx"]) < TOL
    last = R.block_backward(x64, None, a["du"], a["dx_post"], dict(pre_w=up(pre_w), pre_b=None), "rms", "none", eps, 1.0)
    assert rms_off(a["dx"], last["dx"]) < 1e-5 and rms_off(a["d_pre_w"], last["d_pre_w"]) < 1e-4
    # the whole chain in 64 bits, from the same routed tokens
    chain = R.block_backward(None, y_want, None, up(dz), p_post, "rms", "channel", eps, alpha)
    du = oracle.bigmac_backward(u32, chain["dy"].astype(np.float32), *w, wl.k)["dx"]
    whole = R.block_backward(x64, None, du, chain["dx"], dict(pre_w=up(pre_w), pre_b=None), "rms", "none", eps, 1.0)
    assert rms_off(a["dx"], whole["dx"]) < TOL


@pytest.mark.parametrize("T", [1, 37, 700])
def test_serving_step(oracle, T):
    d, r, N, k, h, eps = 256, 64, 16, 4, 192, 1e-5
    wl = synth.small(T=T, d=d, r=r, N=N, k=k, h=h)
    data = synth.generate(wl)
    rng = np.random.default_rng(T)
    rows = T * k
    dims = B.dims_of(wl)
    bf = lambda n, scale=1.0: (B.to_device(data[n], B.F32) * scale).to(torch.bfloat16)  # noqa: E731
    weights = {"w_down": bf("w_down")[None], "w_up": bf("w_up")[None], "w1": bf("w1", 8.0), "w2": bf("w2")}
    packed, held = {}, {}
    for n, w in weights.items():
        packed[n] = B.alloc_bytes(B.mx_packed_bytes(*w.shape))
        B.bigmac_mx_pack(*w.shape, B.BF16, w.contiguous(), packed[n])
        held[n] = np.swapaxes(R.quantise(np.swapaxes(up(w), 1, 2).copy())[2], 1, 2)
    wg = B.to_device(data["w_gate"], B.F32)
    f32 = lambda *s, std=1.0, mean=0.0: torch.from_numpy((mean + std * rng.standard_normal(s)).astype(np.float32)).to(DEV)  # noqa: E731
    x = f32(T, d, std=1.5).to(torch.bfloat16)
    pre_w, post_w = f32(d, std=0.2, mean=1.0), f32(d, std=0.2, mean=1.0)
    gate = torch.rand(T, device=DEV)
    pre = B.make_norm_dims(T, d, parts=B.NORM_PRE, eps=eps)
    both = B.make_norm_dims(T, d, B.BF16, B.F32, B.BF16, kind=B.NORM_RMS, gate=B.GATE_TOKEN, eps=eps)
    pre_p, both_p = B.make_norm_params(pre_w=pre_w), B.make_norm_params(post_w=post_w, pre_w=pre_w, gate=gate)
    down, up_dims = B.make_mx_dims(T, 1, d, r, B.BF16), B.make_mx_dims(T, 1, r, d, B.F32)
    new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    o = dict(u=new((T, d), torch.bfloat16), codes=new((T, d // 2), torch.uint8), scales=new((T, B.mx_scale_bytes(d)), torch.uint8), low=new((T, r), torch.bfloat16),
             idx=new((T, k), torch.int32), gates=new((T, k), torch.float32), x_perm=new((rows, r), torch.bfloat16), offsets=new((N + 1,), torch.int32),
             slot=new((rows,), torch.int32), src=new((rows,), torch.int32), o_perm=new((rows, r), torch.bfloat16), y_low=new((T, r), torch.float32),
             codes2=new((T, r // 2), torch.uint8), scales2=new((T, B.mx_scale_bytes(r)), torch.uint8), y=new((T, d), torch.float32),
             z=new((T, d), torch.bfloat16), u2=new((T, d), torch.bfloat16))
    ws = {n: B.alloc_bytes(B.workspace_bytes(dims, kind)) for n, kind in (("route", B.WS_ROUTE), ("dispatch", B.WS_DISPATCH), ("ffn", B.WS_MX_GROUPED_FFN))}

    def step():
        B.bigmac_norm_forward(pre, pre_p, x, None, None, o["u"])
        B.bigmac_route(dims, o["u"], wg, None, o["idx"], o["gates"], None, ws["route"])
        B.bigmac_mx_quantize(T, d, B.BF16, o["u"], o["codes"], o["scales"])
        B.bigmac_mx_product(down, o["codes"], o["scales"], None, packed["w_down"], None, o["low"])
        B.bigmac_dispatch(dims, o["low"], o["idx"], o["x_perm"], o["offsets"], o["slot"], o["src"], ws["dispatch"])
        B.bigmac_mx_grouped_ffn(dims, o["x_perm"], o["offsets"], packed["w1"], packed["w2"], o["o_perm"], ws["ffn"])
        B.bigmac_combine(dims, o["o_perm"], o["slot"], o["gates"], o["y_low"])
        B.bigmac_mx_quantize(T, r, B.F32, o["y_low"], o["codes2"], o["scales2"])
        B.bigmac_mx_product(up_dims, o["codes2"], o["scales2"], None, packed["w_up"], None, o["y"])
        B.bigmac_norm_forward(both, both_p, x, o["y"], o["z"], o["u2"])

    replays_equal_eager(step, o)
    a = {n: up(v) for n, v in o.items()}
    near = lambda got, want, tol: (np.abs(got - want) <= tol).all()  # noqa: E731
    half = R.HALF_STEP["bf16"] * 1.001
    u_want = R.norm(up(x), up(pre_w), None, "rms", eps)
    assert near(a["u"], u_want, half * np.abs(u_want) + 1e-5)
    idx, gates, _ = oracle.route(a["u"].astype(np.float32), data["w_gate"], None, k)
    assert np.array_equal(o["idx"].cpu().numpy(), idx) and near(a["gates"], gates, 1e-5)
    uq = R.quantise(a["u"])[2]
    low_want, size = uq @ held["w_down"][0], np.abs(uq) @ np.abs(held["w_down"][0])
    assert near(a["low"], low_want, half * np.abs(low_want) + 140 * R.U32 * size)            # 64 + 256 / 64 additions, two steps each
    offsets, slot, _ = oracle.permutation(idx, N)
    assert np.array_equal(o["offsets"].cpu().numpy(), offsets) and np.array_equal(o["slot"].cpu().numpy().reshape(T, k), slot)
    assert np.array_equal(a["x_perm"][slot.reshape(-1)], np.repeat(a["low"], k, 0))
    want, limit = R.ffn(a["x_perm"], list(np.diff(offsets)), held["w1"], held["w2"])
    assert near(a["o_perm"], want, limit)
    y_low = (a["o_perm"][slot] * a["gates"][:, :, None]).sum(1)
    assert near(a["y_low"], y_low, 8 * R.U32 * (np.abs(a["o_perm"][slot]) * a["gates"][:, :, None]).sum(1) + 1e-30)
    yq = R.quantise(a["y_low"])[2]
    assert near(a["y"], yq @ held["w_up"][0], 140 * R.U32 * (np.abs(yq) @ np.abs(held["w_up"][0])) + 1e-30)
    z_want = R.block_forward(up(x), a["y"], dict(post_w=up(post_w), post_b=None, gate=up(gate)), "rms", "token", eps, 1.0)
    assert near(a["z"], z_want, half * np.abs(z_want) + 1e-5)
    u2_want = R.norm(a["z"], up(pre_w), None, "rms", eps)
    assert near(a["u2"], u2_want, half * np.abs(u2_want) + 1e-5)
