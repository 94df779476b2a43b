"""The distillation loss on the GPU against float64 from the whole logits. Bounds: linear_time_ref.distill's."""
import math

import pytest
import torch

from gpu_util import say
from linear_time_ref import distill
from long_context_ref import HALF, check
from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def inputs(T, D, V, K, dtype, seed, hard=True, weights=False, ragged=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    ldw = (V + 63) // 64 * 64
    W = rn(D, ldw) * (2.0 / math.sqrt(D))
    t = dict(h=rn(T, D).to(DT[dtype]), W=W.to(DT[dtype]), values=rn(T, K) * 3,
             index=torch.stack([torch.randperm(V, generator=g, device="cuda")[:K] for _ in range(T)]).int())
    if V > 64:                                       # several of a row in one group of 64 columns, the last columns among them
        t["index"][::3, 0] = V - 1
    if ragged:
        n = torch.randint(0, K + 1, (T, 1), generator=g, device="cuda")
        t["index"].masked_fill_(torch.arange(K, device="cuda") >= n, -1)
        t["values"][::5, 0] = -math.inf
    t["targets"] = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32) if hard else None
    t["weights"] = None
    if weights:
        t["weights"] = torch.rand(T, generator=g, device="cuda") * (torch.rand(T, generator=g, device="cuda") > 0.3) / T
    return t


def config(t, V, **kw):
    T, D = t["h"].shape
    kw.setdefault("dtype", "bf16" if t["h"].dtype == torch.bfloat16 else "f32")
    return bpt.make_distill_config(T, D, V, t["values"].shape[1], **kw)


def run(t, cfg, dloss=1.0):
    d = bpt.DistillLoss(cfg)
    loss, tokens, saved = d.forward(t["h"], t["W"], t["values"], t["index"], t["targets"], t["weights"])
    dh, dW = d.backward(t["h"], t["W"], saved, dloss)
    torch.cuda.synchronize()
    return dict(loss=loss, tokens=tokens, dh=dh, dW=dW)


def compare(t, cfg, out, dloss=1.0):
    ref = distill(t["h"], t["W"], cfg.V, t["values"], t["index"], cfg.tau, cfg.soft, cfg.hard, t["targets"], t["weights"], dloss,
                  HALF[t["h"].dtype], HALF[out["dW"].dtype])
    for name in ("tokens", "loss", "dh", "dW"):
        check(out[name].cpu(), ref[name], ref[name + "_err"], name)


CASES = [
    # T, D, V, K, tau, soft, hard, weights, ragged, kw
    (1, 64, 1, 1, 1.0, 1.0, 0.0, False, False, {}),
    (1, 64, 65, 3, 2.0, 1.0, 1.0, False, False, {}),
    (7, 64, 100, 5, 0.5, 0.7, 0.3, True, True, {}),
    (65, 128, 1000, 8, 1.0, 0.5, 0.5, False, True, {}),
    (130, 192, 513, 64, 4.0, 1.0, 0.0, True, False, {}),
    (200, 64, 4097, 65, 1.0, 1.0, 0.0, False, True, {}),
    (300, 256, 777, 256, 2.0, 0.9, 0.1, True, True, {}),
    (257, 128, 640, 33, 1.5, 1.0, 0.4, False, False, dict(block_rows=100)),
    (520, 64, 300, 20, 3.0, 1.0, 0.4, True, True, dict(block_rows=256)),
    (64, 64, 200, 200, 1.0, 0.0, 1.0, False, False, {}),      # hard targets alone
    (600, 192, 3001, 16, 2.0, 1.0, 0.2, True, True, dict(ldw=3200)),
    # logits formed again in the backward; kept for the first block, the first two of them alone
    (1, 64, 65, 3, 2.0, 1.0, 1.0, False, False, dict(keep_bytes=-1)),
    (130, 192, 513, 64, 4.0, 1.0, 0.0, True, True, dict(keep_bytes=-1)),
    (300, 256, 777, 256, 2.0, 0.9, 0.1, True, True, dict(keep_bytes=-1)),
    (257, 128, 640, 33, 1.5, 1.0, 0.4, False, True, dict(block_rows=100, keep_bytes=100 * 640 * 4)),
    (257, 128, 640, 33, 1.0, 1.0, 0.4, False, True, dict(block_rows=100, keep_bytes=256 * 640 * 4)),
    (1100, 64, 9000, 20, 2.0, 1.0, 0.4, True, True, {}),      # four tiles of a workgroup of the kept logits
    # columns of a last round of tiles in a product of their own
    (300, 64, 33000, 40, 2.0, 1.0, 0.3, True, True, {}),
    (257, 128, 32900, 9, 1.0, 1.0, 0.0, False, True, dict(keep_bytes=-1)),
]


@pytest.mark.parametrize("dtype,grad", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:7])))
def test_loss_and_gradients(case, dtype, grad):
    T, D, V, K, tau, soft, hard, weights, ragged, kw = case
    say(f"case distill {case} {dtype} {grad}")
    t = inputs(T, D, V, K, dtype, T + V, hard > 0, weights, ragged)
    if "ldw" in kw:
        t["W"] = torch.cat([t["W"], torch.randn(D, kw["ldw"] - t["W"].shape[1], device="cuda").to(t["W"].dtype)], 1)
    cfg = config(t, V, tau=tau, soft=soft, hard=hard, grad_dtype=grad, **kw)
    compare(t, cfg, run(t, cfg))


@pytest.mark.parametrize("keep", [0, -1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_upstream_gradient_and_no_dw(dtype, keep):
    t = inputs(90, 64, 333, 12, dtype, 1)
    cfg = config(t, 333, tau=2.0, soft=0.6, hard=0.4, keep_bytes=keep)
    out = run(t, cfg, -2.5)
    compare(t, cfg, out, -2.5)
    d = bpt.DistillLoss(cfg)
    _, _, saved = d.forward(t["h"], t["W"], t["values"], t["index"], t["targets"])
    dh, dW = d.backward(t["h"], t["W"], saved, -2.5, want_dW=False)
    assert dW is None and torch.equal(dh, out["dh"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_index_given_twice(dtype):
    """Counts with the sum of its probabilities: also three times, all the same, and where it is the target."""
    T, V, K = 40, 150, 9
    t = inputs(T, 64, V, K, dtype, 2)
    t["index"][:, 3] = t["index"][:, 0]
    t["index"][::2, 7] = t["index"][::2, 0]
    t["index"][5] = 77
    t["targets"][::4] = t["index"][::4, 0]
    cfg = config(t, V, tau=1.3, soft=1.0, hard=0.5)
    compare(t, cfg, run(t, cfg))


@pytest.mark.parametrize("K", [63, 64, 128, 190, 256])
def test_lists_longer_than_the_vocabulary(K):
    """Ten logits: most indices of a list are given many times, in one row all of them the same; the target is one more entry."""
    T, V = 21, 10
    t = inputs(T, 64, 300, K, "f32", 12)
    t["W"][:, V:] = 0.0
    g = torch.Generator(device="cuda").manual_seed(13)
    t["index"] = torch.randint(-1, V + 1, (T, K), generator=g, device="cuda", dtype=torch.int32)
    t["index"][4] = 3
    t["targets"] = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    cfg = config(t, V, tau=1.5, soft=1.0, hard=0.5, ldw=t["W"].shape[1])
    compare(t, cfg, run(t, cfg))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_order_of_a_list_changes_only_roundings(dtype):
    T, V, K = 33, 500, 70
    t = inputs(T, 64, V, K, dtype, 3)
    cfg = config(t, V, soft=1.0, hard=0.5)
    a = run(t, cfg)
    order = torch.randperm(K, device="cuda")
    t["values"], t["index"] = t["values"][:, order].contiguous(), t["index"][:, order].contiguous()
    b = run(t, cfg)
    compare(t, cfg, b)
    check(b["dh"].cpu(), a["dh"].cpu().double(), 2 * distill(t["h"], t["W"], V, t["values"], t["index"], 1.0, 1.0, 0.5, t["targets"],
                                                             half=HALF[t["h"].dtype])["dh_err"], "dh")


@pytest.mark.parametrize("keep", [0, -1])
@pytest.mark.parametrize("dtype,grad", [("bf16", "bf16"), ("f32", "f32")])
def test_tokens_that_are_left_out(dtype, grad, keep):
    """No weight, or neither list nor target: nothing of them reaches losses or gradients, NaN and infinity in h, in the values or in an
    index of the padding included."""
    T, V, K = 150, 400, 10
    t = inputs(T, 64, V, K, dtype, 4, weights=True)
    t["weights"] = t["weights"] + 1.0 / T
    out = torch.zeros(T, dtype=torch.bool, device="cuda")
    out[::3] = True
    t["weights"][::6] = 0.0
    t["index"][3::6], t["targets"][3::6] = -1, -100
    cfg = config(t, V, tau=2.0, soft=0.5, hard=0.5, grad_dtype=grad, keep_bytes=keep)
    ref = run(t, cfg)
    compare(t, cfg, ref)
    t["h"][::6], t["h"][3::6] = math.nan, math.inf
    t["values"][::6], t["values"][3::6] = math.nan, math.inf
    t["index"][::6], t["targets"][::6] = 2 ** 31 - 1, -2 ** 31
    got = run(t, cfg)
    for k in ref:
        assert torch.equal(got[k], ref[k]), k
    assert bool((got["dh"][out] == 0).all()) and bool((got["tokens"][:, out] == 0).all())


def test_all_tokens_left_out():
    t = inputs(20, 64, 100, 4, "bf16", 5)
    t["weights"] = torch.zeros(20, device="cuda")
    out = run(t, config(t, 100, soft=1.0, hard=1.0))
    assert all(bool((v == 0).all()) for v in out.values())


@pytest.mark.parametrize("keep", [0, -1])
def test_large_logits(keep):
    """Logits of some hundreds: exponentials far below the smallest number, sums against the running maximum."""
    for dtype in ("bf16", "f32"):
        t = inputs(50, 64, 700, 6, dtype, 6)
        t["h"] = (t["h"].float() * 100).to(DT[dtype])
        t["values"] *= 100
        cfg = config(t, 700, tau=0.5, soft=1.0, hard=1.0, keep_bytes=keep)
        compare(t, cfg, run(t, cfg))


def test_blocks_give_the_same_losses():
    """dh and the losses of a token do not hang on the block it is in."""
    t = inputs(300, 128, 1000, 16, "bf16", 7)
    a = run(t, config(t, 1000, tau=2.0, soft=0.5, hard=0.5))
    b = run(t, config(t, 1000, tau=2.0, soft=0.5, hard=0.5, block_rows=77))
    for k in ("loss", "tokens", "dh"):
        assert torch.equal(a[k], b[k]), k


def test_a_large_vocabulary():
    """Pieces of a token's table, 1024 groups of 64 logits each."""
    for dtype in ("bf16", "f32"):
        t = inputs(5, 64, 140001, 40, dtype, 10, ragged=True)
        t["index"][:, 1], t["index"][:, 2], t["index"][:, 3] = 65535, 65536, 131072
        cfg = config(t, 140001, tau=2.0, soft=1.0, hard=0.5)
        compare(t, cfg, run(t, cfg))


@pytest.mark.parametrize("keep", [1 << 34, -1])
def test_offsets_past_32_bits(keep):
    """A block of more than 2^31 logits. Some tokens count, those behind that limit among them: what they give hangs on no other."""
    T, D, V, K = 45056, 64, 50257, 8
    g = torch.Generator(device="cuda").manual_seed(11)
    t = dict(h=torch.randn(T, D, generator=g, device="cuda").bfloat16(),
             W=(torch.randn(D, 50304, generator=g, device="cuda") / 4).bfloat16(), values=torch.randn(T, K, generator=g, device="cuda") * 3,
             index=torch.randint(0, V, (T, K), generator=g, device="cuda", dtype=torch.int32),
             targets=torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32), weights=torch.zeros(T, device="cuda"))
    some = torch.cat([torch.arange(0, T, 4501), torch.arange(T - 12, T)]).cuda()
    t["weights"][some] = 1.0 / len(some)
    cfg = config(t, V, tau=1.5, soft=1.0, hard=0.5, block_rows=T, keep_bytes=keep)
    out = run(t, cfg)
    left = torch.ones(T, dtype=torch.bool, device="cuda")
    left[some] = False
    assert bool((out["dh"][left] == 0).all()) and bool((out["tokens"][:, left] == 0).all())
    few = {k: v if k == "W" else v[some].contiguous() for k, v in t.items()}
    compare(few, cfg, dict(out, dh=out["dh"][some], tokens=out["tokens"][:, some]))


def test_hard_targets_are_the_cross_entropy():
    """soft = 0: bpt_xent's loss and gradients."""
    T, D, V = 260, 128, 900
    t = inputs(T, D, V, 4, "bf16", 8)
    out = run(t, config(t, V, soft=0.0, hard=1.0, grad_dtype="f32"))
    x = bpt.LMHeadLoss(bpt.make_xent_config(T, D, V))
    loss, lse = x.forward(t["h"], t["W"], t["targets"])
    dh, dW = x.backward(t["h"], t["W"], t["targets"], lse)
    ref = distill(t["h"], t["W"], V, t["values"], t["index"], 1.0, 0.0, 1.0, t["targets"], half=HALF[torch.bfloat16])
    for k, v in (("loss", loss), ("dh", dh), ("dW", dW)):
        a = out[k][:1] if k == "loss" else out[k]
        err = ref[k + "_err"][:1] if k == "loss" else ref[k + "_err"]
        check(a.cpu(), v.cpu().double(), 2 * err, k)


@pytest.mark.parametrize("keep", [0, 200 * 1024 * 4, -1])
def test_replays_from_a_graph(keep):
    T, D, V, K = 500, 64, 1000, 20
    t = inputs(T, D, V, K, "bf16", 9, weights=True, ragged=True)
    cfg = config(t, V, tau=2.0, soft=0.5, hard=0.5, block_rows=200, grad_dtype="bf16", keep_bytes=keep)
    ref = run(t, cfg)
    o = dict(loss=torch.empty(3, device="cuda"), tokens=torch.empty(2, T, device="cuda"), dh=torch.empty_like(t["h"]),
             dW=torch.empty_like(t["W"]))
    saved = torch.empty(bpt.distill_saved_bytes(cfg), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(bpt.distill_workspace_bytes(cfg, k) for k in (False, True)), dtype=torch.uint8, device="cuda")

    def step():
        bpt.distill_fwd(cfg, t["h"], t["W"], t["values"], t["index"], o["loss"], o["tokens"], saved, ws, t["targets"], t["weights"])
        bpt.distill_bwd(cfg, t["h"], t["W"], saved, 1.0, o["dh"], o["dW"], ws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        for v in list(o.values()) + [saved, ws]:     # nothing of an earlier call is read
            v.fill_(55)
        graph.replay()
        torch.cuda.synchronize()
        for k in ref:
            assert torch.equal(o[k], ref[k]), k
        eager = run(t, cfg)
        for k in ref:
            assert torch.equal(eager[k], ref[k]), k
