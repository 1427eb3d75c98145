"""The loop of several samples over a shared prompt runs, and its last token is that of the frame kernel over the same tokens."""
from __future__ import annotations

import pytest

from paper_2601_04359_b200 import samples


@pytest.mark.gpu
@pytest.mark.parametrize("grid,page,n,tokens", [((6, 7), 16, 3, 2), ((9, 15), 64, 8, 1)])
def test_loop(grid, page, n, tokens):
    r = samples.generate(samples=n, frames=2, tokens=tokens, grid=grid, heads=(24, 8), page=page, n_text=37, reps=1)
    frame = grid[0] * grid[1]
    assert r["prompt"] == 37 + frame and r["own"] == 2 * (frame + tokens)
    assert r["bytes_apart"] - r["bytes"] == (n - 1) * r["prompt"] * 4096
    # Either kernel rounds its queries, keys (here twice at most) and probabilities to bf16: 2^-8 of each, on logits of unit variance over some hundred keys; outputs below 1 and their own rounding
    assert r["off_frame_kernel"] <= 4 * 2.0 ** -8
