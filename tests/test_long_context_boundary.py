"""Refusals of rotary positions, windowed attention and AdamW over many tensors: every one is made on the host, before
anything is launched (the pointers here are made up)."""
import ctypes
import math
import os

import pytest
import torch

from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.skipif(not os.path.exists(bpt.LIB_PATH), reason="libbpt.so not built")
A = 1 << 20                                          # an aligned address that nothing may touch


def err():
    return bpt.load().bpt_last_error().decode()


# ---------------------------------------------------------------- rotary positions
def rope(**kw):
    c = bpt.make_rope_config(10, 10, 4, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_rope_accepts():
    for c in (rope(), rope(rot=2), rope(rot=62, interleaved=1), rope(pos0=-5), rope(scaling=1, factor=2.0),
              rope(scaling=3, factor=2.0, orig_len=100), rope(dtype=0), rope(dh=128, H=2, rot=128)):
        assert bpt.rope_validate(c) == 0, err()


@pytest.mark.parametrize("kw,code", [
    (dict(rows=0), 1), (dict(S=0), 1), (dict(H=0), 1), (dict(dh=0), 1), (dict(rot=0), 1), (dict(rot=7), 1), (dict(rot=66), 1),
    (dict(rot=-2), 1), (dict(ldx=255), 1), (dict(ldy=64), 1), (dict(ldx=260), 2), (dict(dh=68, ldx=272, ldy=272), 2),
    (dict(dh=256, ldx=1024, ldy=1024, rot=130), 2), (dict(theta=0.0), 1), (dict(theta=math.inf), 1), (dict(theta=math.nan), 1),
    (dict(mscale=math.nan), 1), (dict(scaling=4), 1), (dict(scaling=-1), 1), (dict(scaling=1, factor=0.5), 1),
    (dict(scaling=1, factor=math.nan), 1), (dict(scaling=2, rot=2, factor=2.0), 1), (dict(scaling=3, factor=2.0), 1),
    (dict(scaling=3, factor=2.0, orig_len=9, beta_fast=1.0), 1), (dict(interleaved=2), 1), (dict(reserved=1), 1), (dict(dtype=5), 1),
    (dict(rows=1 << 40), 2), (dict(pos0=1 << 60), 2), (dict(H=1 << 62), 2), (dict(ldx=1 << 50), 2),
])
def test_rope_refuses(kw, code):
    c = rope(**kw)
    assert bpt.rope_validate(c) == code and err()
    assert bpt.load().bpt_rope_fwd(ctypes.byref(c), None, A, 2 * A, None) == code


def test_rope_refuses_pointers():
    lib, c = bpt.load(), rope()
    for fn in (lib.bpt_rope_fwd, lib.bpt_rope_bwd):
        for args in ((None, None, A), (None, A, None), (None, A + 8, A), (None, A, A + 4), (A + 2, A, 2 * A)):
            assert fn(ctypes.byref(c), *args, None) == 1, args
        assert fn(None, None, A, A, None) == 1
        assert fn(ctypes.byref(rope(ldx=512)), None, A, A, None) == 1      # in place with two strides


# ---------------------------------------------------------------- attention
def attn(**kw):
    q, k = torch.empty(2, 10, 4, 64, dtype=torch.bfloat16), torch.empty(2, 30, 2, 64, dtype=torch.bfloat16)
    c = bpt.attn_config_of(q, k, k, q, window=8, sinks=2)
    for name, v in kw.items():
        o, f = name.split("_") if "_" in name else (None, name)
        setattr(getattr(c, o) if o else c, f, v)
    return c


def test_attn_accepts():
    for c in (attn(), attn(window=0, sinks=0), attn(causal=0), attn(sinks=1000), attn(k_sb=0), attn(k_sh=0, v_sh=0), attn(q_st=0)):
        assert bpt.attn_validate(c) == 0, err()
        assert bpt.attn_workspace_bytes(c, True) > 0


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), 1), (dict(Sq=0), 1), (dict(Skv=0), 1), (dict(Hq=0), 1), (dict(Hkv=0), 1), (dict(dh=0), 1), (dict(Hq=3), 1),
    (dict(dh=32), 2), (dict(dh=256), 2), (dict(window=-1), 1), (dict(sinks=-1), 1), (dict(window=0), 1), (dict(scale=0.0), 1),
    (dict(scale=-1.0), 1), (dict(scale=math.nan), 1), (dict(scale=math.inf), 1), (dict(causal=2), 1), (dict(dtype=3), 1),
    (dict(reserved=1), 1), (dict(q_st=260), 1), (dict(k_sb=4), 1), (dict(v_sh=-64), 1), (dict(o_st=64), 1), (dict(o_sb=0), 1),
    (dict(o_sh=8), 1), (dict(q_st=1 << 22), 2), (dict(k_sb=1 << 41), 2), (dict(Sq=1 << 29), 2), (dict(Skv=1 << 40), 2),
    (dict(window=1 << 30), 2), (dict(B=70000), 2), (dict(Hq=70000), 2), (dict(B=60000, Skv=1 << 20), 2),
])
def test_attn_refuses(kw, code):
    c = attn(**kw)
    assert bpt.attn_validate(c) == code, err()
    assert bpt.attn_workspace_bytes(c, False) == 0 and bpt.attn_workspace_bytes(c, True) == 0
    lib = bpt.load()
    p = [i * A for i in range(1, 12)]
    assert lib.bpt_attn_fwd(ctypes.byref(c), p[0], p[1], p[2], None, None, p[3], p[4], p[5], 1 << 30, None) == code
    assert lib.bpt_attn_bwd(ctypes.byref(c), *p[:3], None, None, *p[3:9], p[9], 1 << 30, None) == code


def test_attn_refuses_lengths_beyond_a_launch():
    # fp32: workgroups of 512 threads for every 16 rows and every 16 keys, in one launch of fewer than 2^32 threads
    small = dict(B=1, Hq=1, Hkv=1, q_sb=1 << 36, k_sb=1 << 36, v_sb=1 << 36, o_sb=1 << 36, q_st=64, k_st=64, v_st=64, o_st=64,
                 q_sh=64, k_sh=64, v_sh=64, o_sh=64, dtype=bpt.BPT_F32)
    assert bpt.attn_validate(attn(Sq=2 ** 26 - 16, Skv=2 ** 26, **small)) == 0, err()
    assert bpt.attn_validate(attn(Sq=2 ** 26, Skv=2 ** 26, **small)) == 2
    small["dtype"] = bpt.BPT_BF16
    assert bpt.attn_validate(attn(Sq=2 ** 26, Skv=2 ** 26, **small)) == 0, err()
    small.update({k: 128 for k in small if k.endswith(("_st", "_sh"))}, dh=128)
    assert bpt.attn_validate(attn(Sq=2 ** 28 - 64, Skv=2 ** 28, **small)) == 0, err()
    assert bpt.attn_validate(attn(Sq=2 ** 28, Skv=2 ** 28, **small)) == 2


def test_attn_refuses_pointers():
    lib, c = bpt.load(), attn()
    need = bpt.attn_workspace_bytes(c, True)
    p = [i * A for i in range(1, 11)]

    def fwd(i=None, to=None, ws=p[9], nb=1 << 30, lens=(None, None)):
        a = list(p)
        if i is not None:
            a[i] = to
        return lib.bpt_attn_fwd(ctypes.byref(c), a[0], a[1], a[2], *lens, a[3], a[4], ws, nb, None)

    def bwd(i=None, to=None, nb=1 << 30):
        a = list(p)
        if i is not None:
            a[i] = to
        return lib.bpt_attn_bwd(ctypes.byref(c), *a[:3], None, None, *a[3:9], a[9], nb, None)

    for i in range(5):
        assert fwd(i, None) == 1 and fwd(i, A + 8) == 1
    assert fwd(3, p[0]) == 1 and fwd(3, p[2]) == 1                       # O is an input
    assert fwd(lens=(A + 4, None)) == 1 and fwd(lens=(None, A + 4)) == 1
    for i in list(range(6)) + [7, 8, 9]:
        assert bwd(i, None) == 1, i
    for i in range(10):
        assert bwd(i, A + 8) == 1
    assert bwd(6, p[0]) == 1 and bwd(7, p[5]) == 1 and bwd(8, p[7]) == 1
    assert bwd(nb=need - 1) == 3 and "workspace" in err()
    for o in ("q", "k", "v"):                                            # gradients of broadcast inputs
        s = attn(**{f"{o}_sb": 0})
        assert lib.bpt_attn_bwd(ctypes.byref(s), *p[:3], None, None, *p[3:9], p[9], 1 << 30, None) == 1
        assert "overlap" in err()


def test_attn_config_of_refuses():
    q, k = torch.empty(2, 10, 4, 64), torch.empty(2, 30, 2, 64)
    for args in ((q, k, k[:, :5], q), (q, k[:1], k[:1], q), (q, k, k, q[:, :5]), (q, k.bfloat16(), k, q),
                 (q.half(), k.half(), k.half(), q.half()), (q[0], k, k, q), (q.transpose(2, 3), k, k, q)):
        with pytest.raises((ValueError, TypeError)):
            bpt.attn_config_of(*args)


def test_few_queries_are_cut_along_the_keys():
    """A workspace is asked for exactly where the keys are cut; never more than 64 slices."""
    for dt in (torch.float32, torch.bfloat16):
        one = torch.empty(1, 1, 8, 128, dtype=dt)
        for L, cut in ((64, False), (100000, True)):
            k = torch.empty(1, L, 1, 128, dtype=dt, device="meta")
            n = bpt.attn_workspace_bytes(bpt.attn_config_of(one, k, k, one), False)
            assert (n > 0) == cut and n <= 64 * 8 * (128 * 4 + 8) + 512
        k = torch.empty(1, 100000, 1, 128, dtype=dt, device="meta")
        assert bpt.attn_workspace_bytes(bpt.attn_config_of(one, k, k, one, window=64, sinks=4), False) == 0


# ---------------------------------------------------------------- AdamW
def adam(cfg=None, tensors=None, count=None):
    c = bpt.AdamWMultiConfig(1e-3, 0.9, 0.95, 1e-8, 1, 0, 8, 0, 1, 0)
    for k, v in (cfg or {}).items():
        setattr(c, k, v)
    ts = []
    for j, t in enumerate(tensors if tensors is not None else [{}]):
        x = bpt.AdamWTensor(10, *[A * (10 * j + i) for i in range(1, 7)], 0.1)
        for k, v in t.items():
            setattr(x, k, v)
        ts.append(x)
    arr = (bpt.AdamWTensor * max(1, len(ts)))(*ts)
    return bpt.load().bpt_adamw_multi(ctypes.byref(c), arr, len(ts) if count is None else count, None)


@pytest.mark.parametrize("kw", [
    dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=math.nan), dict(eps=0.0), dict(eps=1e-60), dict(eps=1e-40), dict(eps=math.inf),
    dict(lr=-1.0), dict(lr=math.inf), dict(lr=math.nan), dict(state_bits=16), dict(reserved=1), dict(grad_dtype=2), dict(lowp_dtype=-1),
])
def test_adamw_refuses_configs(kw):
    assert adam(kw) == 1 and err()


@pytest.mark.parametrize("t", [
    dict(n=-1), dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(exps=None), dict(p=A + 4), dict(m=A + 8), dict(v=A + 1),
    dict(p_lowp=A + 2), dict(exps=A + 1), dict(weight_decay=-0.1), dict(weight_decay=math.nan),
])
def test_adamw_refuses_tensors(t):
    assert adam(tensors=[{}, t]) == 1 and err()


def test_adamw_refuses_the_same_tensor_twice():
    assert adam(tensors=[dict(p=A), dict(p=A)]) == 1 and "overlap" in err()
    assert adam(tensors=[dict(p=A, n=100), dict(p=A + 384)]) == 1


def test_adamw_refuses_a_tensor_beyond_a_launch():
    assert adam(tensors=[dict(n=2 ** 33 + 1)]) == 2 and "2^33" in err()


def test_adamw_refuses_counts():
    assert adam(count=-1) == 1
    assert bpt.load().bpt_adamw_multi(None, None, 0, None) == 1
    c = bpt.AdamWMultiConfig(1e-3, 0.9, 0.95, 1e-8, 1, 0, 8, 0, 1, 0)
    assert bpt.load().bpt_adamw_multi(ctypes.byref(c), None, 3, None) == 1
    assert bpt.load().bpt_adamw_multi(ctypes.byref(c), None, 0, None) == 0       # nothing to do
    assert adam(tensors=[dict(n=0, p=None)]) == 0
    arr = (bpt.AdamWTensor * 1)()
    assert bpt.load().bpt_adamw_multi(ctypes.byref(c), arr, 1 << 40, None) == 2


def test_adamw_tensors_refuses():
    p, b = torch.zeros(300), torch.zeros(300, dtype=torch.uint8)
    good = dict(p=p, g=p, m=p, v=p)
    bpt.AdamWTensors([good])
    for bad in (dict(good, m=b), dict(good, g=p.half()), dict(good, v=p[:5]), dict(good, p=torch.zeros(600)[::2]),
                dict(good, p_lowp=p.half())):
        with pytest.raises(ValueError):
            bpt.AdamWTensors([bad])
    with pytest.raises(ValueError):
        bpt.AdamWTensors([dict(p=p, g=p, m=b, r=b, exps=torch.zeros(2, 2, dtype=torch.uint8)[:1])], bits=8)
    with pytest.raises(ValueError):
        bpt.AdamWTensors([good], bits=16)
    with pytest.raises(ValueError):
        bpt.AdamWTensors([good, dict(good, g=p.bfloat16())])
    with pytest.raises(ValueError):
        bpt.adamw_multi(bpt.AdamWTensors([good]), 1, 1e-3)              # on the CPU
    with pytest.raises(ValueError):
        bpt.AdamWTensors([dict(good, m=torch.zeros(300, device="meta"))])


def test_lengths_and_positions_are_int32_on_the_gpu():
    c, q = attn(), torch.empty(2, 10, 4, 64, dtype=torch.bfloat16)
    lse = torch.empty(2, 4, 10)
    for bad in (torch.zeros(2, dtype=torch.int64), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)):
        with pytest.raises(ValueError):
            bpt.attn_fwd(c, q, q, q, q, lse, None, bad)
        with pytest.raises(ValueError):
            bpt.attn_fwd(c, q, q, q, q, lse, None, None, bad)
        with pytest.raises(ValueError):
            bpt.rope_fwd(rope(), q, q, bad)
    with pytest.raises(ValueError):
        bpt.WindowAttention().forward(q, q, q)


# ---------------------------------------------------------------- a layer's options
@pytest.mark.parametrize("kw,code", [
    (dict(), 0), (dict(rot=64), 0), (dict(window=100, sinks=4), 0), (dict(rot=16, window=1), 0), (dict(rot=63), 1), (dict(rot=128), 1),
    (dict(rot=-2), 1), (dict(rot=64, theta=0.0), 1), (dict(rot=64, scaling="linear", factor=0.1), 1), (dict(rot=64, scaling="by_parts"), 1),
    (dict(sinks=4), 1), (dict(window=-1), 1), (dict(window=4, sinks=-1), 1), (dict(window=1 << 40), 2),
])
def test_layer_options(kw, code):
    cfg = bpt.make_config(1, 512, 256, 4, 1024, 128, 128, dtype="bf16")
    o = bpt.make_layer_options(**kw)
    assert bpt.layer_options_validate(cfg, o) == code, err()
    lib = bpt.load()
    if code:
        p = bpt.Params(*([A] * 12))
        assert lib.bpt_layer_fwd_options(ctypes.byref(cfg), ctypes.byref(o), A, ctypes.byref(p), 2 * A, 3 * A, 4 * A, 1 << 40, None) == code
        assert lib.bpt_layer_bwd_options(ctypes.byref(cfg), ctypes.byref(o), A, ctypes.byref(p), 3 * A, 2 * A, 5 * A,
                                         ctypes.byref(bpt.Grads()), 4 * A, 1 << 40, None) == code


def test_layer_options_null():
    cfg = bpt.make_config(1, 512, 256, 4, 1024, 128, 128, dtype="bf16")
    lib, p = bpt.load(), bpt.Params(*([A] * 12))
    assert lib.bpt_layer_options_validate(ctypes.byref(cfg), None) == 1
    assert lib.bpt_layer_fwd_options(ctypes.byref(cfg), None, A, ctypes.byref(p), 2 * A, 3 * A, 4 * A, 1 << 40, None) == 1
    assert lib.bpt_layer_bwd_options(ctypes.byref(cfg), None, A, ctypes.byref(p), 3 * A, 2 * A, 5 * A, None, 4 * A, 1 << 40, None) == 1
    cfg.H = 3                                        # the layer's own refusals come first
    assert lib.bpt_layer_options_validate(ctypes.byref(cfg), ctypes.byref(bpt.make_layer_options())) == 1
