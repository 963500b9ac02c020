"""Host-only checks of window attention's and the optimiser's C ABI: sizes, and arguments that are refused before anything is launched."""
import ctypes
import os

import pytest
import torch

from paper_2503_06671_amd import binding

OK, E_NULL, E_SHAPE, E_DTYPE, E_UNSUP, E_WS, E_ALIAS, E_HIP = range(8)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2503_06671_amd import build
        build.build()
    return binding.load_library()


def attn(**kw):
    a = dict(N=2, H=16, W=16, heads=4, kv_heads=2, head_dim=16, win_h=8, win_w=8, scale=0.25, q_stride=64 * 256, k_stride=32 * 256, v_stride=32 * 256,
             bias=0x9000000, n_edges=0, edges=None, mask=None)
    a.update(kw)
    return binding._WindowAttn(**a)


Q, K, V, OUT, SAVED, GO, GQ, GK, GV, WS = (0x10000000 * i for i in range(1, 11))
BIG = 1 << 26


def test_forward_rejects_bad_arguments_before_launch(lib):
    # the device "pointers" are fake: every call below must fail in validation
    def fw(q=Q, k=K, v=V, dt=0, out=OUT, saved=None, saved_bytes=0, a=None, **kw):
        return lib.esc_window_attention_forward(q, k, v, dt, ctypes.byref(a or attn(**kw)), out, saved, saved_bytes, None)
    for n in ("q", "k", "v", "out"):
        assert fw(**{n: None}) == E_NULL, n
    assert lib.esc_window_attention_forward(Q, K, V, 0, None, OUT, None, 0, None) == E_NULL
    assert fw(dt=2) == E_DTYPE
    for n in ("N", "H", "W", "heads", "kv_heads", "head_dim", "win_h", "win_w"):
        assert fw(**{n: 0}) == E_SHAPE, n
    assert fw(kv_heads=3) == E_SHAPE
    assert fw(head_dim=65) == E_UNSUP
    assert fw(heads=1025, kv_heads=1) == E_UNSUP
    assert fw(win_h=8193) == E_UNSUP
    assert fw(H=65536, W=65536) == E_UNSUP
    assert fw(H=65, W=65, win_h=65, win_w=65, q_stride=BIG, k_stride=BIG, v_stride=BIG) == E_UNSUP   # 129 * 129 offsets
    assert fw(scale=0.0) == fw(scale=-1.0) == fw(scale=float("nan")) == fw(scale=float("inf")) == E_SHAPE
    assert fw(scale=65.0) == fw(scale=2.0 ** -21) == E_UNSUP
    assert fw(q_stride=64 * 256 - 1) == fw(k_stride=-5) == fw(v_stride=1) == E_SHAPE
    assert fw(q=Q + 2) == fw(out=OUT + 1) == fw(bias=0x9000002) == E_SHAPE
    three = (ctypes.c_int * 3)(1, 2, 2)
    at = ctypes.cast(three, ctypes.c_void_p)
    assert fw(n_edges=3, edges=at) == E_SHAPE             # they increase
    three[0] = 0
    assert fw(n_edges=2, edges=at) == E_SHAPE             # and are positive
    assert fw(n_edges=2, edges=None) == E_NULL
    assert fw(n_edges=33, edges=at) == E_UNSUP and fw(n_edges=-1) == E_SHAPE
    assert fw(out=Q) == fw(out=K + 4) == fw(out=V + 2 * 32 * 256 * 4 - 4) == E_ALIAS
    assert fw(mask=OUT + 64) == fw(bias=OUT + 64) == E_ALIAS
    a = attn()
    need = lib.esc_window_attention_saved_bytes(ctypes.byref(a), 0)
    assert need >= 2 * 4 * 256 * 4 and need % 256 == 0
    assert lib.esc_window_attention_saved_bytes(ctypes.byref(a), 1) >= need + 2 * 64 * 256 * 2
    assert lib.esc_window_attention_saved_bytes(ctypes.byref(a), 2) == 0
    assert lib.esc_window_attention_saved_bytes(ctypes.byref(attn(head_dim=0)), 0) == 0
    assert lib.esc_window_attention_saved_bytes(None, 0) == 0
    assert fw(saved=SAVED, saved_bytes=need - 1) == fw(saved=SAVED + 128, saved_bytes=need) == E_WS
    assert fw(saved=OUT + 256, saved_bytes=need) == fw(saved=Q, saved_bytes=need) == E_ALIAS


def test_backward_rejects_bad_arguments_before_launch(lib):
    a0 = attn()
    saved = lib.esc_window_attention_saved_bytes(ctypes.byref(a0), 0)
    need = lib.esc_window_attention_backward_workspace_bytes(ctypes.byref(a0))
    assert need >= 2 * 4 * 256 * 4 and need % 256 == 0
    assert lib.esc_window_attention_backward_workspace_bytes(None) == 0
    assert lib.esc_window_attention_backward_workspace_bytes(ctypes.byref(attn(kv_heads=3))) == 0

    def bw(q=Q, k=K, v=V, dt=0, out=OUT, go=GO, sv=SAVED, svb=saved, gq=GQ, gk=GK, gv=GV, gqs=64 * 256, gks=32 * 256, gvs=32 * 256, gb=None, ws=WS, wsb=need,
           **kw):
        g = binding._WindowGrads(gq, gk, gv, gqs, gks, gvs, gb)
        return lib.esc_window_attention_backward(q, k, v, dt, ctypes.byref(attn(**kw)), out, go, sv, svb, ctypes.byref(g), 0, ws, wsb, None)
    for n in ("q", "k", "v", "out", "go", "sv", "gq", "gk", "gv"):
        assert bw(**{n: None}) == E_NULL, n
    assert lib.esc_window_attention_backward(Q, K, V, 0, ctypes.byref(a0), OUT, GO, SAVED, saved, None, 0, WS, need, None) == E_NULL
    assert bw(gb=0xb0000000, bias=None) == E_NULL         # a gradient of a bias that is not there
    assert bw(dt=3) == E_DTYPE
    assert bw(gqs=5) == bw(gks=-1) == bw(gv=GV + 2) == bw(go=GO + 1) == bw(gb=0xb0000001) == E_SHAPE
    assert bw(svb=saved - 1) == bw(sv=SAVED + 8) == bw(ws=None) == bw(ws=WS + 16) == bw(wsb=need - 256) == E_WS
    assert bw(gq=Q) == bw(gk=GO) == bw(gv=OUT) == bw(gk=GQ) == bw(gv=GK + 512) == bw(gq=SAVED) == bw(gq=WS) == E_ALIAS
    assert bw(gb=WS) == bw(gb=GQ) == bw(gb=0x9000000) == bw(gb=Q) == bw(ws=Q) == bw(ws=SAVED) == E_ALIAS
    # parts of one tensor that interleave are refused only where they meet
    step = 128 * 256
    assert bw(gq=GQ, gk=GQ + 64 * 256 * 4, gv=GQ + 95 * 256 * 4, gqs=step, gks=step, gvs=step) == E_ALIAS
    assert bw(gq=GQ, gk=GQ + 64 * 256 * 4, gv=GQ + 97 * 256 * 4, gqs=step, gks=step, gvs=step) == E_ALIAS   # into the next image's first
    assert bw(gq=GQ, gk=GQ + 64 * 256 * 4, gv=GQ + 96 * 256 * 4, gqs=step, gks=step, gvs=step, wsb=0) == E_WS


def test_launches_and_sizes_have_limits(lib):
    # a lane count of 2^32 and more, sizes in bytes beyond 64 bits: refused, not cut off
    big = 1 << 30
    def sizes(**kw):
        a = attn(**kw)
        return lib.esc_window_attention_saved_bytes(ctypes.byref(a), 0), lib.esc_window_attention_backward_workspace_bytes(ctypes.byref(a))
    tiny = dict(H=1, W=1, heads=1, kv_heads=1, head_dim=1, win_h=1, win_w=1, q_stride=1, k_stride=1, v_stride=1)
    assert sizes(N=(1 << 26) - 64, **tiny) > (0, 0)
    assert sizes(N=1 << 26, **tiny)[1] == 0
    a = attn(N=1 << 26, **tiny)
    assert lib.esc_window_attention_forward(Q, Q + (big << 4), Q + (big << 5), 0, ctypes.byref(a), Q + (big << 6), None, 0, None) == E_UNSUP
    assert sizes(N=(1 << 31) - 1, H=46340, W=46340, heads=1024, kv_heads=1, head_dim=64, win_h=1, win_w=1) == (0, 0)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("head_dim", [16, 32, 64])
def test_windows_up_to_the_limit_have_a_plan(lib, head_dim, dt):
    # whatever a window's shape, up to 16384 offsets; one wavefront or many (a workspace that is too small is found after the plans)
    for h in [*range(1, 65), 100, 333, 1000, 1365, 2000, 2730, 4096, 8192]:
        w = (16384 // (2 * h - 1) + 1) // 2
        for win in {(h, w), (w, h), (h, max(1, w - 1)), (h, max(1, w // 2))}:
            if min(win) < 1 or max(win) > 8192:
                continue
            for N in (1, 64):
                pixels = win[0] * win[1]
                a = attn(N=N, H=win[0], W=win[1], heads=1, kv_heads=1, head_dim=head_dim, win_h=win[0], win_w=win[1],
                         q_stride=pixels * head_dim, k_stride=pixels * head_dim, v_stride=pixels * head_dim)
                far = [0x1000000000 * i for i in range(1, 10)]
                g = binding._WindowGrads(*far[:3], *[pixels * head_dim] * 3, None)
                assert lib.esc_window_attention_backward_workspace_bytes(ctypes.byref(a)) > 0, (win, N)
                assert lib.esc_window_attention_backward(*far[3:6], dt, ctypes.byref(a), far[6], far[7], far[8], 1 << 34, ctypes.byref(g), 0,
                                                         None, 0, None) == E_WS, (win, N)


def test_binding_refuses(lib):
    x = torch.zeros(1, 4, 8, 8)
    with pytest.raises(TypeError, match="device tensor"):
        binding.window_attention_forward(x, x, x, 2, (4, 4))
    with pytest.raises(ValueError):
        binding.new_window_attention_saved(1, 0, 16, 8, 8, torch.float32)
    with pytest.raises(ValueError):
        binding.new_window_attention_backward_workspace(1, 2, 65, 8, 8, (4, 4))
    with pytest.raises(TypeError, match="params"):
        binding.AdamW([torch.zeros(3)], [torch.zeros(3)])
    with pytest.raises(ValueError, match="states"):
        binding.AdamW([torch.zeros(3)], [torch.zeros(3)], states="4bit")
    with pytest.raises(ValueError):
        binding.AdamW([], [])


def tensors(*rows):
    t = (binding._AdamwTensor * len(rows))()
    for i, r in enumerate(rows):
        d = dict(param=0x10000000 + 0x1000000 * i, grad=0x20000000 + 0x1000000 * i, m=0x30000000 + 0x1000000 * i, v=0x40000000 + 0x1000000 * i,
                 m_scale=0x50000000 + 0x1000000 * i, v_scale=0x60000000 + 0x1000000 * i, n=1000, weight_decay=0.1)
        d.update(r)
        for k, x in d.items():
            setattr(t[i], k, x)
    return t


def test_adamw_rejects_bad_arguments_before_launch(lib):
    plan = binding._AdamwPlan()
    memory = 0x70000000

    def init(*rows, n=None, state=0, dt=0, step=0, mem=memory, nbytes=1 << 20, p=plan):
        rows = rows or ({},)
        t = tensors(*rows)
        return lib.esc_adamw_plan_init(t, len(rows) if n is None else n, state, dt, step, mem, nbytes, ctypes.byref(p) if p is not None else None, None)
    assert init(n=0) == init(n=-3) == init({"n": -1}) == init(step=-1) == E_SHAPE
    assert lib.esc_adamw_plan_init(None, 1, 0, 0, 0, memory, 1 << 20, ctypes.byref(plan), None) == E_NULL
    assert init(p=None) == E_NULL
    assert init(state=2) == init(dt=2) == E_DTYPE
    assert init({"n": 1 << 60}) == E_UNSUP
    for k in ("param", "grad", "m", "v"):
        assert init({k: None}) == E_NULL, k
        assert init({k: 0x70001002}) == E_SHAPE or k == "grad", k
    assert init({"grad": 0x20000002}) == init({"grad": 0x20000001}, dt=1) == E_SHAPE
    for k in ("m_scale", "v_scale"):
        assert init({k: None}, state=1) == E_NULL
        assert init({k: 0x50000002}, state=1) == E_SHAPE
    for w in (-0.1, float("nan"), float("inf")):
        assert init({"weight_decay": w}) == E_SHAPE
    t = tensors({}, {})
    need = lib.esc_adamw_plan_bytes(t, 2, 0)
    assert need > 0 and need % 256 == 0
    assert lib.esc_adamw_plan_bytes(t, 0, 0) == lib.esc_adamw_plan_bytes(None, 1, 0) == lib.esc_adamw_plan_bytes(t, 2, 7) == 0
    assert init({}, {}, nbytes=need - 1) == init(mem=None) == init(mem=memory + 8) == E_WS
    # a tensor twice, states that meet, a gradient that is also written, the plan's own memory
    assert init({}, {"param": 0x10000000}) == init({}, {"param": 0x10000000 + 3996}) == E_ALIAS
    assert init({}, {"m": 0x40000000}) == init({}, {"grad": 0x10000000}) == init({"v": memory}) == E_ALIAS
    assert init({}, {"v_scale": 0x50000008}, state=1) == E_ALIAS
    assert not plan.memory, "a plan that was refused stays as it was"


def test_adamw_step_rejects_bad_arguments_before_launch(lib):
    def step(plan=None, **kw):
        h = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, grad_scale=1.0, lr_device=None)
        h.update(kw)
        p = dict(memory=0x70000000, bytes=1 << 20, n=1, chunks=1, state=0, grad_dt=0)
        p.update(plan or {})
        return lib.esc_adamw_step(ctypes.byref(binding._AdamwPlan(**p)), ctypes.byref(binding._AdamwHyper(**h)), None)
    nan, inf = float("nan"), float("inf")
    for k in ("beta1", "beta2"):
        assert step(**{k: 1.0}) == step(**{k: -0.1}) == step(**{k: nan}) == E_SHAPE, k
    for k in ("lr", "eps"):
        assert step(**{k: -1e-9}) == step(**{k: nan}) == step(**{k: inf}) == E_SHAPE, k
    assert step(grad_scale=nan) == step(grad_scale=inf) == step(lr_device=0x1002) == E_SHAPE
    assert step({"memory": None}) == step({"memory": 0x70000010}) == step({"bytes": 64}) == E_WS
    assert step({"n": 0}) == step({"chunks": -1}) == E_SHAPE
    assert step({"state": 5}) == step({"grad_dt": 9}) == E_DTYPE
    assert lib.esc_adamw_step(None, None, None) == E_NULL
