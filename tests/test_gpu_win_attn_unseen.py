"""What windowed attention promises about what is not seen: keys that no query of the call sees change nothing, whatever they hold,
in the backward too; a query that sees nothing has O = 0, lse = -inf and dQ = 0 beside queries that see a NaN."""
import math

import pytest
import torch

from gpu_util import say
from long_context_ref import attention, check
from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(B, Sq, Skv, Hq, Hkv, dh, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda").to(DT[dtype])  # noqa: E731
    return rn(B, Sq, Hq, dh), rn(B, Skv, Hkv, dh), rn(B, Skv, Hkv, dh), rn(B, Sq, Hq, dh)


def run(q, k, v, do, q_lens=None, kv_lens=None, **kw):
    nan = lambda t: torch.full_like(t, math.nan)  # noqa: E731
    o, dq, dk, dv = nan(q), nan(q), nan(k), nan(v)
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), math.nan, device="cuda")
    cfg = bpt.attn_config_of(q, k, v, o, **kw)
    ws = torch.full((max(bpt.attn_workspace_bytes(cfg, False), bpt.attn_workspace_bytes(cfg, True)),), 255, dtype=torch.uint8,
                    device="cuda")
    lens = [None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda") for t in (q_lens, kv_lens)]
    bpt.attn_fwd(cfg, q, k, v, o, lse, ws, *lens)
    bpt.attn_bwd(cfg, q, k, v, o, lse, do, dq, dk, dv, ws, *lens)
    torch.cuda.synchronize()
    return {"O": o, "lse": lse, "dQ": dq, "dK": dk, "dV": dv}


ROLLING = [
    # B, Sq, Skv, Hq, Hkv, causal, window, sinks
    (1, 100, 900, 4, 2, True, 50, 3),
    (2, 100, 900, 4, 2, False, 50, 0),
    (1, 1, 300, 2, 1, True, 20, 2),
    (1, 65, 260, 3, 1, True, 1, 0),
    (1, 300, 2500, 8, 1, True, 50, 4),               # chunks
    (4, 600, 1100, 16, 8, True, 40, 5),              # sinks apart
    (3, 300, 1200, 16, 8, False, 64, 70),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("case", ROLLING, ids=lambda s: "-".join(str(int(x)) for x in s))
def test_keys_that_a_rolling_cache_gave_up(case, dh, dtype):
    """A piece of a prompt behind a long cache: what lies between the sinks and the first query's window holds NaN and infinity, and
    gets zero gradients."""
    B, Sq, Skv, Hq, Hkv, causal, window, sinks = case
    say(f"case rolling {case} dh {dh} {dtype}")
    q, k, v, do = make(B, Sq, Skv, Hq, Hkv, dh, dtype, Skv)
    gone = Skv - Sq - window + 1
    assert gone > sinks
    k[:, sinks:gone:2], k[:, sinks + 1:gone:2] = math.nan, math.inf
    v[:, sinks:gone:3], v[:, sinks + 1:gone:3], v[:, sinks + 2:gone:3] = math.inf, math.nan, -math.inf
    kw = dict(causal=causal, window=window, sinks=sinks)
    got = run(q, k, v, do, **kw)
    ref, err = attention(q, k, v, do, **kw)
    for n in ref:
        check(got[n], ref[n], err[n], n)
    assert not bool(got["dK"][:, sinks:gone].any()) and not bool(got["dV"][:, sinks:gone].any())


BLIND = [
    # B, Sq, Skv, Hq, Hkv, causal, window, sinks: queries in front of the first key see nothing
    (1, 20, 10, 2, 1, True, 0, 0),                   # few rows
    (1, 1200, 1100, 1, 1, True, 0, 0),               # few rows in slices
    (8, 300, 130, 16, 8, True, 0, 0),
    (8, 300, 130, 16, 8, True, 20, 3),
    (2, 130, 50, 2, 1, False, 9, 2),
    (4, 700, 650, 16, 8, True, 33, 7),               # sinks apart
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("case", BLIND, ids=lambda s: "-".join(str(int(x)) for x in s))
def test_queries_that_see_nothing_beside_a_nan(case, dh, dtype):
    """The first keys, which the blind queries' neighbours see, hold NaN (V) and infinity (K)."""
    B, Sq, Skv, Hq, Hkv, causal, window, sinks = case
    say(f"case blind {case} dh {dh} {dtype}")
    q, k, v, do = make(B, Sq, Skv, Hq, Hkv, dh, dtype, Sq)
    k[:, 0], k[:, 1], v[:, 0], v[:, 2] = math.inf, math.nan, math.nan, math.inf
    blind = Sq - Skv - (0 if causal else window - 1)
    if sinks and not causal:
        blind = 0                                    # sinks are seen by all
    got = run(q, k, v, do, causal=causal, window=window, sinks=sinks)
    assert not bool(got["O"][:, :blind].any()) and not bool(got["dQ"][:, :blind].any())
    assert bool((got["lse"][:, :, :blind] == -math.inf).all()) and not bool((got["lse"][:, :, blind:] == -math.inf).any())
