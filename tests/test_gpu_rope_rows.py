"""Rotary positions of more rows than a launch holds (2^26 rows, four to a workgroup of 256 threads, are 2^32 threads)."""
import pytest
import torch

from gpu_util import say
from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.gpu
ROWS, PIECE = 2 ** 26 + 5, 2 ** 24


@pytest.mark.parametrize("layout,S", [("half", ROWS), ("interleaved", ROWS), ("half", 1000), ("half", 2 ** 25 + 12345), ("half", 1)])
def test_rows_beyond_a_launch(layout, S):
    """2^26 + 5 rows of 8 features (1 GiB), in runs of S positions: the bits that pieces of 2^24 rows with given positions
    have, forward, and backward in place; and with given positions as a whole."""
    say(f"case rope {ROWS} rows, runs of {S}, {layout}")
    X = torch.empty(ROWS, 8, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for r in range(0, ROWS, PIECE):
        X[r:r + PIECE].copy_(torch.randn(min(PIECE, ROWS - r), 8, generator=g, device="cuda"))
    whole = bpt.make_rope_config(ROWS, S, 1, 8, layout=layout, pos0=7)
    assert bpt.rope_validate(whole) == 0
    pos = (torch.arange(ROWS, device="cuda") % S + 7).int()
    Y, P = torch.full_like(X, float("nan")), torch.full_like(X, float("nan"))
    bpt.rope_fwd(whole, X, Y)
    bpt.rope_fwd(whole, X, P, pos)
    assert torch.equal(Y, P)
    Z = X.clone()
    bpt.rope_bwd(whole, Z, Z)
    for r in range(0, ROWS, PIECE):
        n = min(PIECE, ROWS - r)
        cfg = bpt.make_rope_config(n, n, 1, 8, layout=layout)
        want = torch.empty(n, 8, dtype=torch.bfloat16, device="cuda")
        bpt.rope_fwd(cfg, X[r:r + n], want, pos[r:r + n])
        assert torch.equal(Y[r:r + n], want), r
        bpt.rope_bwd(cfg, X[r:r + n], want, pos[r:r + n])
        assert torch.equal(Z[r:r + n], want), r
