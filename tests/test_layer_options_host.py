"""What a layer and a GPT refuse of their options before anything is allocated or launched (on the CPU)."""
import os

import pytest
import torch

from paper_2305_19370_amd import bpt
from paper_2305_19370_amd.gpt import GPT, GPTShape

pytestmark = pytest.mark.skipif(not os.path.exists(bpt.LIB_PATH), reason="libbpt.so not built")


def test_qkv_grads_with_a_window_are_refused_first():
    cfg = bpt.make_config(1, 64, 256, 4, 512, 64, 64, dtype="f32", out_dtype="f32")
    lay = bpt.Layer(cfg, device="meta", options=bpt.make_layer_options(rot=64, window=16))
    x = torch.empty(1, 64, 256, device="meta")
    with pytest.raises(ValueError, match="window"):
        lay.backward(x, {}, x, x, qkv_grads=True)


SHAPE = dict(L=1, B=1, S=64, D=256, H=4, F=512, V=100, Bq=64, Bkv=64, dtype="f32")


@pytest.mark.parametrize("kw", [
    dict(sinks=4), dict(rope_scaling="linear", rope_factor=2.0), dict(rope_factor=2.0), dict(rope_orig_len=100), dict(window=-1),
    dict(window=16, sinks=-1), dict(opt_bits=16), dict(rope="half", rope_scaling="linear", rope_factor=0.5),
])
def test_gpt_refuses(kw):
    """A setting that nothing would read, or that the layer refuses."""
    with pytest.raises((ValueError, bpt.BptError)):
        GPT(GPTShape(**SHAPE, **kw), device="cpu", init=False)


def test_gpt_takes_what_belongs_together():
    for kw in (dict(), dict(window=16), dict(window=16, sinks=4), dict(rope="half", rope_scaling="linear", rope_factor=2.0),
               dict(rope="interleaved", rope_scaling="by_parts", rope_factor=2.0, rope_orig_len=64, window=8), dict(opt_bits=8)):
        m = GPT(GPTShape(**SHAPE, **kw), device="cpu", init=False)
        assert (m.options is not None) == bool(kw.keys() & {"window", "rope"})
