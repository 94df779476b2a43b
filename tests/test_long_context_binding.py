"""What the Python binding checks before a long-context operator is called: every tensor against the configuration. On the CPU,
where each refusal is told from the last one (a tensor that is not on the GPU) by what it names."""
import os

import pytest
import torch

from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.skipif(not os.path.exists(bpt.LIB_PATH), reason="libbpt.so not built")
BF = torch.bfloat16


def packed(B=2, S=10, Hq=4, Hkv=2, dh=64, dtype=BF):
    x = torch.zeros(B, S, Hq + 2 * Hkv, dh, dtype=dtype)
    return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]


def strided(t):
    """A tensor of t's strides, in memory of its own."""
    return torch.empty_strided(t.shape, t.stride(), dtype=t.dtype)


@pytest.fixture
def call():
    """The tensors of a call on columns of one projection, all as the configuration has them."""
    q, k, v = packed()
    o = torch.empty(q.shape, dtype=BF)
    lse = torch.empty(2, 4, 10)
    ws = torch.empty(1 << 20, dtype=torch.uint8)
    return bpt.attn_config_of(q, k, v, o, window=4, sinks=1), dict(
        q=q, k=k, v=v, o=o, lse=lse, do=torch.empty_like(o), dq=strided(q), dk=strided(k), dv=strided(v), workspace=ws)


FWD = ("q", "k", "v", "o", "lse", "workspace")


def test_only_the_place_is_left_to_refuse(call):
    cfg, t = call
    with pytest.raises(ValueError, match="on the GPU"):
        bpt.attn_fwd(cfg, **{n: t[n] for n in FWD})
    with pytest.raises(ValueError, match="on the GPU"):
        bpt.attn_bwd(cfg, **t)
    t["dq"] = None
    with pytest.raises(ValueError, match="on the GPU"):
        bpt.attn_bwd(cfg, **t)


@pytest.mark.parametrize("name,bad", [
    ("q", lambda t: t[:, :9]), ("q", lambda t: t.contiguous()), ("q", lambda t: t.float()), ("k", lambda t: t.contiguous()),
    ("v", lambda t: t.transpose(1, 2)), ("o", lambda t: t[:, :, :3]), ("o", lambda t: t.float()),
    ("lse", lambda t: t[:, :, :9].contiguous()), ("lse", lambda t: t.to(BF)), ("lse", lambda t: t.double()),
    ("lse", lambda t: t.transpose(1, 2)),
    ("do", lambda t: t.float()), ("do", lambda t: t[:1]), ("do", lambda t: torch.empty(2, 4, 10, 64, dtype=BF).transpose(1, 2)),
    ("dq", torch.Tensor.contiguous), ("dk", torch.Tensor.contiguous), ("dv", torch.Tensor.contiguous),   # empty_like of a view is dense
    ("dq", lambda t: t.float()), ("dk", lambda t: t[:, :5]), ("dv", lambda t: t.half()),
])
def test_attention_refuses(call, name, bad):
    cfg, t = call
    t[name] = bad(t[name])
    with pytest.raises(ValueError, match=f"^{name} must"):
        bpt.attn_bwd(cfg, **t)
    if name in FWD:
        with pytest.raises(ValueError, match=f"^{name} must"):
            bpt.attn_fwd(cfg, **{n: t[n] for n in FWD})


# ---------------------------------------------------------------- rotary positions
def rope_cfg(**kw):
    return bpt.make_rope_config(12, 4, 2, 64, **kw)


GOOD = [
    lambda: torch.empty(12, 2, 64, dtype=BF), lambda: torch.empty(12, 128, dtype=BF), lambda: torch.empty(3, 4, 2, 64, dtype=BF),
    lambda: torch.empty(3, 4, 128, dtype=BF), lambda: torch.empty(12 * 128, dtype=BF), lambda: torch.empty(3, 4, 1, 2, 64, dtype=BF),
]
WIDE = [
    lambda: torch.empty(12, 400, dtype=BF), lambda: torch.empty(12, 400, dtype=BF)[:, :128].view(12, 2, 64),
    lambda: torch.empty(3, 4, 400, dtype=BF)[..., :128], lambda: torch.empty(3, 4, 400, dtype=BF)[..., :128].unflatten(2, (2, 64)),
    lambda: torch.empty(12, 400, dtype=BF)[:, 16:144], lambda: torch.empty(11 * 400 + 128, dtype=BF),
]
BAD = [
    lambda: torch.empty(12, 2, 64), lambda: torch.empty(12, 2, 64, dtype=torch.half), lambda: torch.empty(11, 2, 64, dtype=BF),
    lambda: torch.empty(12, 1, 64, dtype=BF), lambda: torch.empty(2, 12, 64, dtype=BF).transpose(0, 1),
    lambda: torch.empty(12, 120, dtype=BF), lambda: torch.empty(12 * 128 - 1, dtype=BF), lambda: torch.empty(24, 128, dtype=BF)[::2],
    lambda: torch.empty(3, 5, 128, dtype=BF)[:, :4], lambda: torch.empty(12, 256, dtype=BF)[:, ::2],
]


@pytest.mark.parametrize("fn", [bpt.rope_fwd, bpt.rope_bwd])
def test_rope_tensors(fn):
    a, b = ("X", "Y") if fn is bpt.rope_fwd else ("dY", "dX")
    ok = torch.empty(12, 2, 64, dtype=BF)
    for make in GOOD:
        for args in ((make(), ok), (ok, make())):
            with pytest.raises(ValueError, match="on the GPU"):
                fn(rope_cfg(), *args)
    for make in BAD + [w for w in WIDE if make_is_wide(w)]:
        with pytest.raises(ValueError, match=f"^{a} must"):
            fn(rope_cfg(), make(), ok)
        with pytest.raises(ValueError, match=f"^{b} must"):
            fn(rope_cfg(), ok, make())
    wide = rope_cfg(ldx=400, ldy=400)
    for make in WIDE:
        with pytest.raises(ValueError, match="on the GPU"):
            fn(wide, make(), make())
    for make in GOOD:
        with pytest.raises(ValueError, match=f"^{a} must"):
            fn(wide, make(), WIDE[0]())


def make_is_wide(make):
    """All but the flat buffer, which is long enough for rows side by side too."""
    return make().dim() > 1


def test_rope_of_one_row():
    cfg = bpt.make_rope_config(1, 1, 2, 64, ldx=400)
    for x in (torch.empty(1, 2, 64, dtype=BF), torch.empty(128, dtype=BF), torch.empty(2, 64, dtype=BF), torch.empty(1, 400, dtype=BF)):
        with pytest.raises(ValueError, match="on the GPU"):
            bpt.rope_fwd(cfg, x, torch.empty(1, 2, 64, dtype=BF))
