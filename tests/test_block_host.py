"""Host-only checks of the layer norm's, the point-wise product's and dropout's C ABI: sizes, and arguments that are refused before anything is launched."""
import ctypes
import os

import pytest
import torch

from paper_2503_06671_amd import binding

OK, E_NULL, E_SHAPE, E_DTYPE, E_UNSUP, E_WS, E_ALIAS, E_HIP = range(8)
X, OUT, GO, SKIP, GX, SAVED, WS, W, B, GW, GB = (0x10000000 * i for i in range(1, 12))  # no memory: every call below must fail in validation
BIG = 1 << 27
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2503_06671_amd import build
        build.build()
    return binding.load_library()


def norm(**kw):
    a = dict(N=2, C=8, H=5, W=7, eps=1e-5, weight=W, bias=B, x_stride=280, out_stride=280, skip_stride=280)
    a.update(kw)
    return binding._LayerNorm(**a)


def test_layernorm_forward_rejects(lib):
    def fw(x=X, dt=0, out=OUT, saved=None, saved_bytes=0, **kw):
        return lib.esc_layernorm_forward(x, dt, ctypes.byref(norm(**kw)), out, saved, saved_bytes, None)
    assert fw(x=None) == fw(out=None) == lib.esc_layernorm_forward(X, 0, None, OUT, None, 0, None) == E_NULL
    assert fw(dt=2) == fw(dt=-1) == E_DTYPE
    for n in ("N", "C", "H", "W"):
        assert fw(**{n: 0}) == fw(**{n: -4}) == E_SHAPE, n
    assert fw(eps=0.0) == fw(eps=-1e-5) == fw(eps=NAN) == fw(eps=INF) == E_SHAPE
    assert fw(C=65537) == fw(H=65536, W=32768) == fw(N=1 << 20, H=1024, W=1024) == E_UNSUP
    assert fw(x_stride=279) == fw(out_stride=-1) == fw(out_stride=0) == fw(x_stride=(1 << 46) + 1) == E_SHAPE
    assert fw(x=X + 2) == fw(out=OUT + 1) == fw(weight=W + 2) == fw(bias=B + 1) == fw(dt=1, x=X + 1) == E_SHAPE
    assert fw(out=X) == fw(out=X + 4 * 559) == fw(out=X - 4 * 559) == fw(weight=OUT + 32) == fw(bias=OUT + 4 * 559) == E_ALIAS
    need = lib.esc_layernorm_saved_bytes(ctypes.byref(norm()))
    assert need == 768 and need == lib.esc_layernorm_saved_bytes(ctypes.byref(norm(C=100, eps=0)))
    assert lib.esc_layernorm_saved_bytes(None) == lib.esc_layernorm_saved_bytes(ctypes.byref(norm(H=0))) == 0
    assert fw(saved=SAVED, saved_bytes=need - 1) == fw(saved=SAVED + 64, saved_bytes=need) == E_WS
    assert fw(saved=X, saved_bytes=need) == fw(saved=OUT + 256, saved_bytes=need) == fw(saved=W - 256, saved_bytes=need) == fw(saved=B, saved_bytes=need) == E_ALIAS


def test_layernorm_backward_rejects(lib):
    need = lib.esc_layernorm_backward_workspace_bytes(ctypes.byref(norm()))
    saved = lib.esc_layernorm_saved_bytes(ctypes.byref(norm()))
    assert need > 0 and need % 256 == 0
    assert lib.esc_layernorm_backward_workspace_bytes(None) == lib.esc_layernorm_backward_workspace_bytes(ctypes.byref(norm(N=0))) == 0

    def bw(x=X, go=GO, skip=SKIP, dt=0, sv=SAVED, svb=saved, gx=GX, gxs=280, gw=GW, gb=GB, ws=WS, wsb=need, **kw):
        g = binding._LayerNormGrads(gx, gxs, gw, gb)
        return lib.esc_layernorm_backward(x, go, skip, dt, ctypes.byref(norm(**kw)), sv, svb, ctypes.byref(g), 0, ws, wsb, None)
    assert bw(x=None) == bw(go=None) == bw(sv=None) == bw(gx=None, gw=None, gb=None) == E_NULL
    assert lib.esc_layernorm_backward(X, GO, None, 0, ctypes.byref(norm()), SAVED, saved, None, 0, WS, need, None) == E_NULL
    assert bw(dt=3) == E_DTYPE
    assert bw(W=0) == E_SHAPE and bw(C=65537) == E_UNSUP
    assert bw(x_stride=3) == bw(out_stride=279) == bw(skip_stride=279) == bw(gxs=279) == E_SHAPE
    assert bw(x=X + 1) == bw(go=GO + 2) == bw(skip=SKIP + 2) == bw(gx=GX + 3) == bw(gw=GW + 2) == bw(gb=GB + 1) == bw(weight=W + 1) == E_SHAPE
    assert bw(svb=saved - 1) == bw(sv=SAVED + 8) == bw(ws=None) == bw(ws=WS + 8) == bw(wsb=need - 1) == E_WS
    assert bw(gx=X) == bw(gx=GO + 4) == bw(gx=SKIP) == bw(gx=SAVED) == bw(gx=W) == bw(gx=WS) == bw(gx=GW) == E_ALIAS
    assert bw(gw=X) == bw(gw=GO) == bw(gw=SKIP + 100) == bw(gw=W) == bw(gw=SAVED) == bw(gw=WS) == bw(gw=GB) == bw(gb=GX) == E_ALIAS
    assert bw(ws=X) == bw(ws=GO) == bw(ws=SAVED) == bw(ws=SKIP) == E_ALIAS


def pointwise(**kw):
    a = dict(N=2, K=8, M=6, H=5, W=7, act=0, w=W, b=B, x_stride=280, out_stride=210, residual_stride=210)
    a.update(kw)
    return binding._Pointwise(**a)


def test_pointwise_forward_rejects(lib):
    def fw(x=X, res=SKIP, dt=0, out=OUT, **kw):
        return lib.esc_pointwise_forward(x, res, dt, ctypes.byref(pointwise(**kw)), out, None)
    assert fw(x=None) == fw(out=None) == fw(w=None) == lib.esc_pointwise_forward(X, None, 0, None, OUT, None) == E_NULL
    assert fw(dt=2) == E_DTYPE
    for n in ("N", "K", "M", "H", "W"):
        assert fw(**{n: 0}) == fw(**{n: -1}) == E_SHAPE, n
    assert fw(act=3) == fw(act=-1) == E_SHAPE
    assert fw(K=65537, x_stride=BIG) == fw(M=65537) == fw(K=32768, M=16384, x_stride=BIG, out_stride=BIG, residual_stride=BIG) == fw(H=65536, W=32768) == fw(N=1 << 20, H=1024, W=1024) == E_UNSUP
    assert fw(x_stride=279) == fw(out_stride=209) == fw(residual_stride=0) == E_SHAPE
    assert fw(x=X + 2) == fw(res=SKIP + 2) == fw(out=OUT + 1) == fw(w=W + 2) == fw(b=B + 3) == E_SHAPE
    assert fw(out=X + 4) == fw(out=SKIP) == fw(w=OUT) == fw(b=OUT + 4 * 419) == fw(out=W + 4 * 47) == E_ALIAS


def test_pointwise_backward_rejects(lib):
    def size(dt=0, **kw):
        return lib.esc_pointwise_backward_workspace_bytes(ctypes.byref(pointwise(**kw)), dt)
    need = size()
    assert need > 0 and need % 256 == 0 and size(act=1) >= need + 2 * 6 * 35 * 4 and size(dt=1) > 0
    assert size(dt=2) == size(N=0) == size(act=5) == lib.esc_pointwise_backward_workspace_bytes(None, 0) == 0

    def bw(x=X, go=GO, dt=0, gx=GX, gxs=280, gw=GW, gb=GB, ws=WS, wsb=None, **kw):
        g = binding._PointwiseGrads(gx, gxs, gw, gb)
        return lib.esc_pointwise_backward(x, go, dt, ctypes.byref(pointwise(**kw)), ctypes.byref(g), 0, ws, size(dt, **kw) if wsb is None else wsb, None)
    assert bw(x=None) == bw(go=None) == bw(w=None) == bw(gx=None, gw=None, gb=None) == E_NULL
    assert lib.esc_pointwise_backward(X, GO, 0, ctypes.byref(pointwise()), None, 0, WS, need, None) == E_NULL
    assert bw(dt=2) == E_DTYPE and bw(act=7) == bw(K=0) == E_SHAPE and bw(M=65537) == E_UNSUP
    assert bw(x_stride=1) == bw(out_stride=209) == bw(gxs=279) == E_SHAPE
    assert bw(x=X + 2) == bw(go=GO + 1) == bw(gx=GX + 2) == bw(gw=GW + 2) == bw(gb=GB + 1) == bw(w=W + 1) == E_SHAPE
    assert bw(ws=None) == bw(ws=WS + 64) == bw(wsb=need - 1) == bw(act=2, wsb=need) == E_WS
    assert bw(gx=X) == bw(gx=GO) == bw(gx=W) == bw(gx=WS) == bw(gx=GW) == bw(gw=W) == bw(gw=X) == bw(gw=GO) == bw(gw=GB) == bw(gb=WS) == bw(ws=X) == E_ALIAS


def drop(**kw):
    a = dict(N=2, C=8, H=5, W=7, p=0.25, over=0, seed=1, offset=2, offset_device=None, x_stride=280, out_stride=280, residual_stride=280)
    a.update(kw)
    return binding._Dropout(**a)


def test_dropout_rejects(lib):
    def fw(x=X, res=SKIP, dt=0, out=OUT, **kw):
        return lib.esc_dropout_forward(x, res, dt, ctypes.byref(drop(**kw)), out, None)

    def bw(go=GO, dt=0, gx=GX, **kw):
        return lib.esc_dropout_backward(go, dt, ctypes.byref(drop(**kw)), gx, None)
    assert fw(x=None) == fw(out=None) == bw(go=None) == bw(gx=None) == E_NULL
    assert lib.esc_dropout_forward(X, None, 0, None, OUT, None) == lib.esc_dropout_backward(GO, 0, None, GX, None) == E_NULL
    assert fw(dt=2) == bw(dt=2) == E_DTYPE
    for n in ("N", "C", "H", "W"):
        assert fw(**{n: 0}) == bw(**{n: -1}) == E_SHAPE, n
    assert fw(over=3) == fw(over=-1) == bw(over=9) == E_SHAPE
    assert fw(p=-0.1) == fw(p=1.0) == fw(p=NAN) == bw(p=INF) == E_SHAPE
    assert fw(p=1 - 2.0 ** -18) == E_UNSUP
    assert fw(H=65536, W=32768) == fw(N=1 << 20, C=1 << 10, H=1 << 10, W=1 << 10, x_stride=1 << 30) == E_UNSUP
    assert fw(x_stride=279) == fw(out_stride=1) == fw(residual_stride=-280) == bw(x_stride=279) == bw(out_stride=279) == E_SHAPE
    assert fw(x=X + 2) == fw(res=SKIP + 1) == fw(out=OUT + 2) == fw(dt=1, out=OUT + 1) == fw(offset_device=0x9000004) == E_SHAPE
    assert fw(out=X) == fw(out=SKIP + 4) == fw(offset_device=OUT + 8) == bw(gx=GO) == bw(gx=GO + 4 * 559) == E_ALIAS


def test_binding_refuses_without_a_gpu():
    x, w = torch.zeros(1, 4, 2, 2), torch.zeros(3, 4)
    with pytest.raises(TypeError):
        binding.layernorm_forward(x)
    with pytest.raises(TypeError):
        binding.pointwise_forward(x, w)
    with pytest.raises(TypeError):
        binding.dropout_forward(x, 0.5, 1)
    with pytest.raises(ValueError):
        binding.pointwise_forward(x, w, act="relu")
    with pytest.raises(ValueError):
        binding.dropout_backward(x, 0.5, 1, over="pixel")
    with pytest.raises(ValueError):
        binding.new_layernorm_saved(0, 1, 1, device="cpu")
    with pytest.raises(ValueError):
        binding.new_layernorm_backward_workspace(1, 0, 1, 1, device="cpu")
    with pytest.raises(ValueError):
        binding.new_pointwise_backward_workspace(1, 4, 0, 1, 1, torch.float32, device="cpu")
    with pytest.raises(ValueError):
        binding.new_pointwise_backward_workspace(1, 4, 4, 1, 1, torch.float32, act="tanh", device="cpu")
    assert binding.new_pointwise_backward_workspace(1, 4, 4, 3, 3, torch.bfloat16, act="gelu", device="cpu").numel() % 256 == 0
