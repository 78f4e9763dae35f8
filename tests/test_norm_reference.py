"""The plain norms of block_reference: gradients against central differences, and the host-side refusals of the library's calls."""
import ctypes

import numpy as np
import pytest

from paper_2502_16927_amd import binding as B
import block_reference as R


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
def test_gradients_against_differences(kind, gate):
    rng = np.random.default_rng(7)
    T, d, eps, alpha = 3, 8, 1e-3, 0.7
    t = {n: rng.standard_normal((T, d)) for n in ("x", "y", "cu", "cz")}
    t.update({n: 1.0 + 0.3 * rng.standard_normal(d) for n in ("post_w", "post_b", "pre_w", "pre_b")})
    t["gate"] = {"none": lambda: None, "channel": lambda: rng.standard_normal(d), "token": lambda: rng.standard_normal(T), "full": lambda: rng.standard_normal((T, d))}[gate]()

    def loss():
        z = R.block_forward(t["x"], t["y"], t, kind, gate, eps, alpha)
        return float((t["cu"] * R.norm(z, t["pre_w"], t["pre_b"], kind, eps)).sum() + (t["cz"] * z).sum())

    z = R.block_forward(t["x"], t["y"], t, kind, gate, eps, alpha)
    got = R.block_backward(z, t["y"], t["cu"], t["cz"], t, kind, gate, eps, alpha)
    step = 1e-5
    for name, grad in (("x", "dx"), ("y", "dy"), ("gate", "d_gate"), ("post_w", "d_post_w"), ("post_b", "d_post_b"), ("pre_w", "d_pre_w"), ("pre_b", "d_pre_b")):
        if t[name] is None:
            assert got[grad] is None
            continue
        for i in np.ndindex(t[name].shape):
            keep = t[name][i]
            t[name][i] = keep + step
            up = loss()
            t[name][i] = keep - step
            down = loss()
            t[name][i] = keep
            # the loss is about 10, its third derivatives about 100: rounding 10 2^-52 / step, cut-off 100 step^2
            assert abs((up - down) / (2 * step) - got[grad][i]) < 1e-6, (name, i)


def dims(**kw):
    return B.make_norm_dims(**{"T": 4, "d": 64, **kw})


def test_workspace_and_bad_dims():
    assert B.norm_workspace_bytes(dims()) > 0 and B.norm_workspace_bytes(dims(T=1 << 20, d=8192)) % 256 == 0
    fake = ctypes.c_void_p(4096)                 # never dereferenced: the dims are checked first
    p = B.NormParams(4096, None, 4096, None, None)
    nan, inf = float("nan"), float("inf")
    for bad, code in ((dict(T=0), -1), (dict(T=-3), -1), (dict(d=0), -1), (dict(d=12), -1), (dict(d=8200), -5), (dict(T=(1 << 30) + 1), -5), (dict(x_dtype=2), -1),
                      (dict(y_dtype=-1), -1), (dict(u_dtype=5), -1), (dict(kind=2), -1), (dict(parts=0), -1), (dict(parts=B.NORM_ACCUMULATE), -1), (dict(parts=11), -1),
                      (dict(gate=4), -1), (dict(gate=-1), -1), (dict(parts=B.NORM_PRE, gate=B.GATE_TOKEN), -1), (dict(eps=-1.0), -1), (dict(eps=nan), -1),
                      (dict(eps=inf), -1), (dict(alpha=inf), -1), (dict(alpha=nan), -1), (dict(parts=B.NORM_PRE, alpha=0.5), -1)):
        d = dims(**bad)
        assert B.norm_workspace_bytes(d) == 0, bad
        assert B.lib().bigmac_norm_forward(ctypes.byref(d), ctypes.byref(p), fake, fake, fake, fake, None) == code, bad
        assert B.lib().bigmac_norm_backward(ctypes.byref(d), ctypes.byref(p), *[fake] * 12, 1 << 40, None) == code, bad
    assert B.lib().bigmac_norm_forward(None, ctypes.byref(p), fake, fake, fake, fake, None) == -1
    assert B.lib().bigmac_norm_forward(ctypes.byref(dims()), None, fake, fake, fake, fake, None) == -1


def test_pointers_that_do_not_go_with_the_parts():
    L, both, pre, post = B.lib(), dims(), dims(parts=B.NORM_PRE), dims(parts=B.NORM_POST)
    P = lambda *a: B.NormParams(*[4096 if v else None for v in a])  # noqa: E731

    def forward(d, p, x=4096, y=4096, z=4096, u=4096):
        return L.bigmac_norm_forward(ctypes.byref(d), ctypes.byref(p), x, y, z, u, None)

    full = P(1, 0, 1, 0, 0)
    for d, p in ((both, P(0, 0, 1, 0, 0)), (both, P(1, 0, 0, 0, 0)), (pre, full), (post, full), (pre, P(0, 1, 1, 0, 0)), (post, P(1, 0, 0, 1, 0)),
                 (both, P(1, 0, 1, 0, 1)), (dims(gate=B.GATE_CHANNEL), full)):
        assert forward(d, p) == -1
    for bad in (dict(x=None), dict(y=None), dict(z=None), dict(u=None), dict(x=4100), dict(y=4104), dict(z=4098), dict(u=4097)):
        assert forward(both, full, **bad) == -1, bad
    assert forward(pre, P(0, 0, 1, 0, 0)) == -1                      # y and z without a branch
    assert forward(post, P(1, 0, 0, 0, 0)) == -1                     # u without its norm
    assert forward(both, B.NormParams(4100, None, 4096, None, None)) == -1

    names = ("z", "y", "du", "dz", "dx", "dy", "d_gate", "d_post_w", "d_post_b", "d_pre_w", "d_pre_b", "ws")

    def backward(d, p, ws_bytes=1 << 40, **kw):
        at = dict(dict.fromkeys(names, 4096), d_gate=None, d_post_b=None, d_pre_b=None)
        at.update(kw)
        return L.bigmac_norm_backward(ctypes.byref(d), ctypes.byref(p), *[at[n] for n in names], ws_bytes, None)

    for bad in (dict(z=None), dict(y=None), dict(du=None), dict(dx=None), dict(dy=None), dict(d_gate=4096), dict(d_post_w=None), dict(d_post_b=4096), dict(d_pre_w=None),
                dict(d_pre_b=4096), dict(ws=None), dict(dx=4104), dict(ws=4097)):
        assert backward(both, full, **bad) == -1, bad
    assert backward(both, full, ws_bytes=B.norm_workspace_bytes(both) - 1) == -2
    none = dict(z=None, du=None, d_pre_w=None)
    assert backward(post, P(1, 0, 0, 0, 0), dz=None, **none) == -1   # nothing to differentiate
    assert backward(both, P(1, 1, 1, 0, 0)) == -1                    # a bias without its gradient


class Weights:
    """Stands for a contiguous tensor on a GPU."""

    def __init__(self, gpu):
        self.gpu, self.device = gpu, f"cuda:{gpu}"

    def get_device(self):
        return self.gpu

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


@pytest.mark.parametrize("name", ["post_w", "post_b", "pre_w", "pre_b", "gate"])
def test_parameters_of_another_gpu_are_refused(name, monkeypatch):
    """Weights, biases and the gate lie on the GPU that is current when they are used, whichever was when they were put together."""
    here = [0]
    monkeypatch.setattr(B.torch.cuda, "current_device", lambda: here[0])
    monkeypatch.setattr(B, "_stream", lambda stream, device=None: None)
    p = B.make_norm_params(**{name: Weights(1)})
    forward = lambda: B.bigmac_norm_forward(dims(), p, None, None, None, None)  # noqa: E731
    backward = lambda: B.bigmac_norm_backward(dims(), p, *[None] * 12)  # noqa: E731
    for call in (forward, backward):
        with pytest.raises(ValueError):
            call()
    here[0] = 1
    for call in (forward, backward):                                 # on to the library's own checks: there is no x
        with pytest.raises(B.BigmacError):
            call()
    with pytest.raises(ValueError):
        B.make_norm_params(**{"pre_w": Weights(0), "post_w": Weights(0), name: Weights(1)}, **({} if name.endswith("_b") else {"post_b": Weights(0)}))
