"""What a layer and a GPT refuse of their options before anything is allocated or launched (on the CPU)."""
import os

import pytest
import torch

from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.skipif(not os.path.exists(bpt.LIB_PATH), reason="libbpt.so not built")


def test_qkv_grads_with_a_window_are_refused_first():
    cfg = bpt.make_config(1, 64, 256, 4, 512, 64, 64, dtype="f32", out_dtype="f32")
    lay = bpt.Layer(cfg, device="meta", options=bpt.make_layer_options(rot=64, window=16))
    x = torch.empty(1, 64, 256, device="meta")
    with pytest.raises(ValueError, match="window"):
        lay.backward(x, {}, x, x, qkv_grads=True)
