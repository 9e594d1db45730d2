"""im2win_linear_attention where weights, rows and elements of a state differ by more than a 16-bit type holds (tolerances: linear_64)."""
import math

import pytest
import torch

from test_gpu_linear_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("segments", [1, 3])
@pytest.mark.parametrize("growth,tokens,scale", [(0.05, 200, 2.0 ** -8), (0.5, 150, 2.0 ** -104)])
def test_decays_that_grow_over_whole_chunks(dtype, segments, growth, tokens, scale, monkeypatch):
    """exp(G_n - G_i) far above 1: the weighted k of a chunk are larger than any k.  (e^10 and e^75 in all; scale brings the last rows into
    the type's range.)"""
    monkeypatch.setenv("IM2WIN_SEGMENTS", str(segments))
    def edit(q, k, v, g, st):
        g.fill_(growth)
    for dk, dv in ((64, 64), (128, 128)):
        run(dtype, [tokens], 2, 1, dk, dv, edit=edit, scale=scale)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("segments", [1, 2])
@pytest.mark.parametrize("decay", [-0.2, -0.3, -0.5, -1.0])
@pytest.mark.parametrize("behind", [0.0, 1e-6])
def test_states_from_the_first_tokens_of_a_chunk(dtype, segments, decay, behind, monkeypatch):
    """k that are 0 or tiny behind the first tokens (gated or masked ones)."""
    monkeypatch.setenv("IM2WIN_SEGMENTS", str(segments))
    def edit(q, k, v, g, st):
        st.zero_()
        g.fill_(decay)
        k[8:64].mul_(behind)
        k[72:].mul_(behind)
    for dk in (64, 128):
        run(dtype, [128], 2, 1, dk, 64, edit=edit)
