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


def test_strides_of_single_elements_count_for_nothing():
    """One sequence, one token: whatever stride such a dimension shows is taken, and is a valid one in the configuration."""
    x = torch.zeros(7 * 5 * 3 * 64 + 8, dtype=BF)
    q = x.as_strided((1, 1, 3, 64), (13, 7, 64, 1))
    k = x.as_strided((1, 5, 3, 64), (3, 192, 64, 1))
    cfg = bpt.attn_config_of(q, k, k, q)
    assert bpt.attn_validate(cfg) == 0
    with pytest.raises(ValueError, match="on the GPU"):
        bpt.attn_fwd(cfg, q, k, k, torch.empty(1, 1, 3, 64, dtype=BF), torch.empty(1, 3, 1), None)


# ---------------------------------------------------------------- rotary positions
def rope_cfg(**kw):
    return bpt.make_rope_config(12, 4, 2, 64, **kw)


GOOD = [
    lambda: torch.empty(12, 2, 64, dtype=BF), lambda: torch.empty(12, 128, dtype=BF), lambda: torch.empty(3, 4, 2, 64, dtype=BF),
    lambda: torch.empty(3, 4, 128, dtype=BF), lambda: torch.empty(12 * 128, dtype=BF), lambda: torch.empty(3, 4, 1, 2, 64, dtype=BF),
    lambda: torch.empty(3, 4 * 128, dtype=BF), lambda: torch.empty(6, 256, dtype=BF),   # rows side by side
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


# ---------------------------------------------------------------- WindowAttention
def test_window_attention_refuses_gradients_of_another_kind():
    q, k, v = packed()
    o, lse = torch.empty(q.shape, dtype=BF), torch.empty(2, 4, 10)
    att = bpt.WindowAttention(window=4)
    for do in (torch.empty(q.shape), torch.empty(2, 9, 4, 64, dtype=BF)):
        with pytest.raises(ValueError, match="^do must"):
            att.backward(q, k, v, o, lse, do)
    with pytest.raises(ValueError, match="^lse must"):
        att.backward(q, k, v, o, lse[:1], torch.empty_like(o))
    with pytest.raises(ValueError, match="on the GPU"):
        att.backward(q, k, v, o, lse, torch.empty_like(o))


def test_gradients_side_by_side():
    """Columns of a projection give columns of one gradient, without a gap; tensors of their own, or of which another is most of the
    rows, do not."""
    q, k, v = packed()
    g = bpt._side_by_side((q, k, v))
    assert [t.stride() for t in g] == [q.stride()] * 3 and [t.shape for t in g] == [q.shape, k.shape, v.shape]
    assert len({t.untyped_storage().data_ptr() for t in g}) == 1 and g[0].untyped_storage().nbytes() == 2 * 2 * 10 * 8 * 64
    assert [t.storage_offset() for t in g] == [0, 256, 384]
    assert [t.storage_offset() for t in bpt._side_by_side((v, q, k))] == [384, 0, 256]
    x = torch.zeros(2, 10, 40, 64, dtype=BF)
    assert bpt._side_by_side((x[:, :, :4], x[:, :, 4:6], x[:, :, 6:8])) is None        # a fifth of the rows
    assert bpt._side_by_side((q, k, k)) is None and bpt._side_by_side((q, k, v.clone())) is None
    assert bpt._side_by_side((q, k, v.contiguous())) is None
    assert bpt._side_by_side((q[:, :, :3], k, v[:, :9])) is None
    y = torch.zeros(2, 10, 8, 72, dtype=BF)
    z = y[..., 4:68]                                                                   # not at 16 bytes
    assert bpt._side_by_side((z[:, :, :4], z[:, :, 4:6], z[:, :, 6:])) is None


def test_what_a_gradient_can_be_laid_out_like():
    x = torch.zeros(2, 10, 4, 64, dtype=BF)
    assert bpt._apart(x) and bpt._apart(x.transpose(1, 2)) and bpt._apart(x[:, :, 1:3]) and bpt._span(x) == x.numel()
    assert bpt._span(x[:, :5]) > x[:, :5].numel()
    assert not bpt._apart(x[:1].expand(2, 10, 4, 64)) and not bpt._apart(x.transpose(2, 3)) and not bpt._apart(x[..., ::2])
    assert not bpt._apart(torch.zeros(2, 10, 4, 68, dtype=BF)[..., 4:])
