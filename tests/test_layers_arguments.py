"""CPU tests of the checks of the linear layer, the embedding and the
optimiser step: in the library (before any HIP call) and in the binding."""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import layers_oracle as orc
from paper_2608_11519_amd import flarepp as fp

_P = [ctypes.c_void_p(i + 1 << 44) for i in range(16)]  # aligned, far apart, never dereferenced: validation fails first
BAD = ctypes.c_void_p(4096 + 8)


@pytest.fixture(autouse=True)
def _lib():
    fp.load()


def _forward(dtype=fp.BF16, act=fp.ACT_GELU, T=100, K=1024, N=32, ptrs=None, ws=_P[15], nbytes=1 << 30):
    return fp.load().flarepp_linear_forward(dtype, act, T, K, N, *(ptrs or _P[:6]), ws, nbytes, None)


def _backward(dtype=fp.BF16, act=fp.ACT_GELU, T=100, K=64, N=32, ptrs=None, ws=_P[15], nbytes=1 << 30):
    return fp.load().flarepp_linear_backward(dtype, act, T, K, N, *(ptrs or _P[:7]), ws, nbytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=0), fp.ERR_INVALID_ARG), (dict(K=0), fp.ERR_INVALID_ARG), (dict(N=-1), fp.ERR_INVALID_ARG),
    (dict(T=(1 << 30) + 1), fp.ERR_UNSUPPORTED), (dict(K=65537), fp.ERR_UNSUPPORTED), (dict(N=65537), fp.ERR_UNSUPPORTED),
    (dict(T=1 << 30, K=2048), fp.ERR_UNSUPPORTED), (dict(dtype=2), fp.ERR_UNSUPPORTED), (dict(act=4), fp.ERR_UNSUPPORTED),
    (dict(act=-1), fp.ERR_UNSUPPORTED), (dict(ws=None), fp.ERR_WORKSPACE), (dict(nbytes=8), fp.ERR_WORKSPACE),
    (dict(ws=BAD), fp.ERR_INVALID_ARG),
])
def test_linear_refuses(kw, code):
    assert _forward(**kw) == code and fp.last_error()
    assert _backward(**kw) == code and fp.last_error()


def test_linear_refuses_pointers():
    for i in range(6):  # X, W, bias, residual, out, pre
        ptrs = list(_P[:6])
        ptrs[i] = BAD
        assert _forward(ptrs=ptrs) == fp.ERR_INVALID_ARG and "aligned" in fp.last_error()
        if i in (0, 1, 4):
            ptrs[i] = None
            assert _forward(ptrs=ptrs) == fp.ERR_INVALID_ARG
    for i, j in ((4, 0), (4, 1), (4, 2), (5, 0), (5, 1), (5, 4), (5, 3)):
        for at in (0, 16, -16):  # the same buffer, or one that reaches into it
            ptrs = list(_P[:6])
            ptrs[i] = ctypes.c_void_p(ptrs[j].value + at)
            assert _forward(ptrs=ptrs) == fp.ERR_INVALID_ARG and "overlap" in fp.last_error()
    ptrs = list(_P[:6])
    ptrs[3] = ctypes.c_void_p(ptrs[4].value + 16)  # in place, but not quite
    assert _forward(ptrs=ptrs) == fp.ERR_INVALID_ARG
    assert _forward(ws=_P[4]) == fp.ERR_INVALID_ARG
    for i in range(7):  # X, W, pre, dOut, dX, dW, dbias
        ptrs = list(_P[:7])
        ptrs[i] = BAD
        assert _backward(ptrs=ptrs) == fp.ERR_INVALID_ARG
        if i < 4:
            ptrs[i] = None
            assert _backward(ptrs=ptrs) == fp.ERR_INVALID_ARG
    assert _backward(ptrs=_P[:4] + [None] * 3) == fp.ERR_INVALID_ARG
    for i in (4, 5, 6):
        for j in range(7):
            ptrs = list(_P[:7])
            ptrs[i] = ptrs[j]
            assert i == j or _backward(ptrs=ptrs) == fp.ERR_INVALID_ARG


def test_linear_workspaces():
    assert fp.flarepp_linear_workspace_bytes(fp.BF16, 0, 64, 64) == 0
    assert fp.flarepp_linear_backward_workspace_bytes(fp.BF16, 9, 64, 64, 64) == 0
    T, K, N = 1000, 128, 256
    # the activation's gradient (two parts with bf16) and the bias sums
    assert fp.flarepp_linear_backward_workspace_bytes(fp.BF16, fp.ACT_GELU, T, K, N) >= 4 * T * N
    assert fp.flarepp_linear_backward_workspace_bytes(fp.F32, fp.ACT_GELU, T, K, N) >= 4 * T * N
    # no workspace where the reduction is not split
    assert fp.flarepp_linear_workspace_bytes(fp.BF16, 100, 64, 32) == 256
    assert fp.flarepp_linear_workspace_bytes(fp.BF16, 100, 1024, 32) > 256
    assert fp.flarepp_embedding_backward_workspace_bytes(100, 5, 8) == 256
    # what is summed per split does not grow with the tokens
    a, b = (fp.flarepp_linear_backward_workspace_bytes(fp.BF16, fp.ACT_NONE, t, K, N) for t in (1 << 18, 1 << 24))
    assert b <= 1.1 * a


def test_embedding_refuses():
    lib = fp.load()
    fwd = lambda dt=fp.BF16, T=10, V=5, C=8, p=_P: lib.flarepp_embedding_forward(dt, T, V, C, p[0], p[1], 1.0, p[2], None)  # noqa: E731
    bwd = lambda dt=fp.BF16, T=10, V=5, C=8, p=_P, ws=_P[9], n=1 << 30: lib.flarepp_embedding_backward(  # noqa: E731
        dt, T, V, C, p[0], p[1], 1.0, p[2], ws, n, None)
    for f in (fwd, bwd):
        for kw in (dict(T=0), dict(V=0), dict(C=0)):
            assert f(**kw) == fp.ERR_INVALID_ARG
        for kw in (dict(dt=5), dict(T=(1 << 30) + 1), dict(V=(1 << 30) + 1), dict(C=65537), dict(V=1 << 30, C=2048)):
            assert f(**kw) == fp.ERR_UNSUPPORTED
        for i in range(3):
            for bad in (None, BAD):
                p = list(_P)
                p[i] = bad
                assert f(p=p) == fp.ERR_INVALID_ARG
        assert f(p=[_P[0], _P[1], _P[1]]) == fp.ERR_INVALID_ARG
    many = dict(T=10000, V=5, C=8)
    assert bwd(ws=None, **many) == fp.ERR_WORKSPACE and bwd(n=64, **many) == fp.ERR_WORKSPACE
    assert fp.flarepp_embedding_backward_workspace_bytes(0, 5, 8) == 0


def _table(count=2, q8=False):
    t = (fp._AdamwTensor * count)()
    for i in range(count):
        t[i].n = 100
        for j, k in enumerate(("p", "g", "m", "v") + (("m_scale", "v_scale") if q8 else ())):
            setattr(t[i], k, (1 << 20) * (1 + i) + 4096 * j)
    return t


def _step(t, state=fp.STATE_F32, count=2, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, step=1, sched=None):
    return fp.load().flarepp_adamw_step(state, count, t, lr, b1, b2, eps, step, sched, None)


@pytest.mark.parametrize("kw,code", [
    (dict(state=2), fp.ERR_UNSUPPORTED), (dict(count=0), fp.ERR_INVALID_ARG), (dict(lr=-1.0), fp.ERR_INVALID_ARG),
    (dict(lr=math.nan), fp.ERR_INVALID_ARG), (dict(lr=math.inf), fp.ERR_INVALID_ARG), (dict(b1=1.0), fp.ERR_INVALID_ARG),
    (dict(b1=-0.1), fp.ERR_INVALID_ARG), (dict(b2=math.nan), fp.ERR_INVALID_ARG), (dict(eps=-1.0), fp.ERR_INVALID_ARG),
    (dict(eps=math.inf), fp.ERR_INVALID_ARG), (dict(step=0), fp.ERR_INVALID_ARG), (dict(step=-3), fp.ERR_INVALID_ARG),
    (dict(step=(1 << 31) + 1), fp.ERR_UNSUPPORTED), (dict(sched=BAD), fp.ERR_INVALID_ARG),
])
def test_adamw_refuses(kw, code):
    assert _step(_table(), **kw) == code and fp.last_error()


def test_adamw_refuses_tensors():
    assert _step(None) == fp.ERR_INVALID_ARG
    for q8 in (False, True):
        state = fp.STATE_E4M3 if q8 else fp.STATE_F32
        for k in ("p", "g", "m", "v") + (("m_scale", "v_scale") if q8 else ()):
            for bad in (None, 4096 + 8):
                t = _table(q8=q8)
                setattr(t[1], k, bad)
                assert _step(t, state=state) == fp.ERR_INVALID_ARG, k
    t = _table(q8=True)  # scales without an 8-bit state
    assert _step(t) == fp.ERR_INVALID_ARG
    for n in (0, -5):
        t = _table()
        t[0].n = n
        assert _step(t) == fp.ERR_INVALID_ARG
    for wd in (-1.0, math.nan, math.inf):
        t = _table()
        t[0].weight_decay = wd
        assert _step(t) == fp.ERR_INVALID_ARG


def test_adamw_refuses_buffers_that_overlap():
    def overlap(k, other, at):
        t = _table()
        setattr(t[1], k, getattr(t[0], other) + at)
        return _step(t)

    for k in ("p", "m", "v", "p_low"):
        for other in ("p", "g", "m", "v"):
            for at in (0, 384):  # the same buffer, its last 16 bytes
                assert overlap(k, other, at) == fp.ERR_INVALID_ARG and "overlap" in fp.last_error(), (k, other, at)
    t = _table()
    t[1].p = t[1].p_low = t[1].p
    assert _step(t) == fp.ERR_INVALID_ARG


def test_schedule():
    s = fp.flarepp_adamw_schedule(lr=0.25, step=3, betas=(0.5, 0.75)).numpy()
    assert s[:8].view(np.float64)[0] == 0.25
    assert s[8:12].view(np.float32)[0] == np.float32(0.25 / (1 - 0.5 ** 3))
    assert s[12:16].view(np.float32)[0] == np.float32(1 / math.sqrt(1 - 0.75 ** 3))
    assert s[16:20].view(np.uint32)[0] == 3
    with pytest.raises(fp.FlareppError):
        fp.flarepp_adamw_schedule(lr=0.25, step=0)


# ---- binding -------------------------------------------------------------------

def _layer(dtype=torch.bfloat16, T=6, K=8, N=5):
    return torch.zeros(2, T // 2, K, dtype=dtype), torch.zeros(K, N, dtype=dtype), torch.zeros(N, dtype=dtype)


def test_linear_binding_checks():
    X, W, b = _layer()
    with pytest.raises(ValueError, match="GPU"):  # consistent: stops at the device
        fp.flarepp_linear_forward(X, W, b, act=fp.ACT_RELU, residual=torch.zeros(2, 3, 5, dtype=X.dtype), keep_pre=True)
    with pytest.raises(TypeError):
        fp.flarepp_linear_forward(X.half(), W.half())
    with pytest.raises(TypeError):
        fp.flarepp_linear_forward(X, W.float())
    with pytest.raises(TypeError):
        fp.flarepp_linear_forward(X, W, b.float())
    with pytest.raises(ValueError):
        fp.flarepp_linear_forward(X, W.t())
    with pytest.raises(ValueError):
        fp.flarepp_linear_forward(X, W, b[:4])
    with pytest.raises(ValueError):
        fp.flarepp_linear_forward(X, W, residual=torch.zeros(6, 5, dtype=X.dtype))
    with pytest.raises(TypeError):
        fp.flarepp_linear_forward(X, W, ws=torch.zeros(100))
    with pytest.raises(TypeError):
        fp.flarepp_linear_forward(X, W, act="gelu")
    d = torch.zeros(2, 3, 5, dtype=X.dtype)
    with pytest.raises(ValueError, match="GPU"):
        fp.flarepp_linear_backward(X, W, d, pre=d, act=fp.ACT_RELU)
    with pytest.raises(ValueError):
        fp.flarepp_linear_backward(X, W, d[:, :2])
    with pytest.raises(TypeError):
        fp.flarepp_linear_backward(X, W, d.float())
    with pytest.raises(TypeError):  # weight gradients are fp32
        fp.flarepp_linear_backward(X, W, d, out={"dW": W.clone()})
    with pytest.raises(ValueError):
        fp.flarepp_linear_backward(X, W, d, out={"dbeta": W.clone()})


def test_embedding_binding_checks():
    ids, table = torch.zeros(4, 3, dtype=torch.int64), torch.zeros(7, 5)
    with pytest.raises(ValueError, match="GPU"):
        fp.flarepp_embedding_forward(ids, table)
    with pytest.raises(TypeError):
        fp.flarepp_embedding_forward(ids.int(), table)
    with pytest.raises(TypeError):
        fp.flarepp_embedding_forward(ids, table.double())
    with pytest.raises(ValueError):
        fp.flarepp_embedding_forward(ids, table[0])
    d = torch.zeros(4, 3, 5)
    with pytest.raises(ValueError, match="GPU"):
        fp.flarepp_embedding_backward(ids, d, V=7)
    with pytest.raises(ValueError):
        fp.flarepp_embedding_backward(ids, d[:, 0], V=7)
    with pytest.raises(TypeError):
        fp.flarepp_embedding_backward(ids, d, V=7.0)
    with pytest.raises(fp.FlareppError):
        fp.flarepp_embedding_backward(ids, d, V=0)
    with pytest.raises(ValueError):
        fp.flarepp_embedding_backward(ids, d, V=7, out=torch.zeros(6, 5))


def test_adamw_binding_checks():
    n = 300
    f32 = lambda: dict(p=torch.zeros(n), g=torch.zeros(n), m=torch.zeros(n), v=torch.zeros(n))  # noqa: E731
    q8 = lambda: dict(p=torch.zeros(n), g=torch.zeros(n), m=torch.zeros(n).to(torch.float8_e4m3fn),  # noqa: E731
                      v=torch.zeros(n).to(torch.float8_e4m3fn), m_scale=torch.zeros(2), v_scale=torch.zeros(2))
    for make in (f32, q8):
        with pytest.raises(ValueError, match="GPU"):
            fp.flarepp_adamw_plan([make(), dict(make(), p_low=torch.zeros(n, dtype=torch.bfloat16), weight_decay=0.1)])
        for bad in (dict(p=torch.zeros(n).bfloat16()), dict(g=torch.zeros(n, dtype=torch.bfloat16)), dict(v=None),
                    dict(p_low=torch.zeros(n))):
            with pytest.raises(TypeError):
                fp.flarepp_adamw_plan([dict(make(), **bad)])
        for bad in (dict(g=torch.zeros(n + 1)), dict(momentum=1)):
            with pytest.raises(ValueError):
                fp.flarepp_adamw_plan([dict(make(), **bad)])
    with pytest.raises(ValueError):
        fp.flarepp_adamw_plan([dict(q8(), m_scale=torch.zeros(1))])
    with pytest.raises(ValueError):
        fp.flarepp_adamw_plan([dict(f32(), m_scale=torch.zeros(2))])
    with pytest.raises(ValueError):
        fp.flarepp_adamw_plan([])
    with pytest.raises(TypeError):
        fp.flarepp_adamw_step([f32()], lr=1e-3, step=1)


# ---- the float64 reference against differences --------------------------------------

@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_reference_slopes_are_the_activations_differences(act):
    y = np.linspace(-6, 6, 2001) + 1e-3
    h = 1e-5
    d = (orc.activate(y + h, act) - orc.activate(y - h, act)) / (2 * h)
    assert np.abs(d - orc.slope(y, act)).max() < 1e-8


def test_reference_backward_against_differences():
    rng = np.random.default_rng(1)
    X, W, b, d = (rng.standard_normal(s) for s in ((5, 4), (4, 3), (3,), (5, 3)))
    pre = orc.linear_forward(X, W, b, None, "gelu")[1]
    dX, dW, db = orc.linear_backward(X, W, pre, d, "gelu")
    f = lambda X, W, b: float((orc.linear_forward(X, W, b, None, "gelu")[0] * d).sum())  # noqa: E731
    h = 1e-6
    for a, g, at in ((X, dX, 0), (W, dW, 1), (b, db, 2)):
        for i in np.ndindex(a.shape):
            e = np.zeros_like(a)
            e[i] = h
            args = [X, W, b]
            up, dn = list(args), list(args)
            up[at], dn[at] = a + e, a - e
            assert abs((f(*up) - f(*dn)) / (2 * h) - g[i]) < 1e-7
