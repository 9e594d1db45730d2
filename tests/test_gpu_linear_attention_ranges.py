"""im2win_linear_attention where weights, rows and elements of a state differ by more than a 16-bit type holds (tolerances: linear_64)."""
import pytest
import torch

from paper_2608_20725_b200 import binding
from sequence_helpers import close, linear_64, sequence_list
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


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("segments", [1, 2])
def test_columns_of_k_that_differ_by_2_to_the_20(dtype, segments, monkeypatch):
    monkeypatch.setenv("IM2WIN_SEGMENTS", str(segments))
    def edit(q, k, v, g, st):
        k[:, :, 0::2].mul_(2.0 ** 10)
        q[:, :, 0::2].mul_(2.0 ** -10)
        k[:, :, 1::2].mul_(2.0 ** -10)
        q[:, :, 1::2].mul_(2.0 ** 10)
        st.zero_()
    for dk in (64, 128):
        run(dtype, [150], 2, 1, dk, 64, edit=edit)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("segments", [1, 2])
@pytest.mark.parametrize("decay", [-0.2, -0.3])
def test_states_whose_later_v_are_zero(dtype, segments, decay, monkeypatch):
    """Columns of v that are 0 behind the first tokens, whose weights are e^-19 of the chunk's largest, where other columns are not."""
    monkeypatch.setenv("IM2WIN_SEGMENTS", str(segments))
    def edit(q, k, v, g, st):
        st.zero_()
        g.fill_(decay)
        v[4:, :, 0::3] = 0.0
    for dk in (64, 128):
        run(dtype, [64], 2, 1, dk, 64, edit=edit)
        run(dtype, [64, 100], 2, 1, dk, 64, edit=edit)


@pytest.mark.parametrize("decay", [-0.5, -1.0, -3.0])
def test_states_whose_later_v_are_zero_behind_any_decay(decay):
    """fp16: what the pieces leave off is 2^-62 of the chunk's largest weighted k, for each v it meets."""
    gen = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(64, 1, 128, generator=gen).half() for _ in range(3))
    v[4:, :, 0::3] = 0.0
    g = torch.full((64, 1), decay)
    o, state = torch.empty(64, 1, 128, dtype=torch.float16, device="cuda"), torch.empty(1, 1, 128, 128, device="cuda")
    ws = binding.alloc_attention_workspace(binding.make_attention_shape(64, 1, 1, 1, 128, 128), torch.float16)
    cu = torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    binding.im2win_linear_attention(q.cuda(), k.cuda(), v.cuda(), g.cuda(), o, ws, state_out=state, cu_seqlens=cu)
    zeros = torch.zeros(1, 1, 128, 128)
    _, _, new, off = linear_64(q, k, v, g, 1.0, torch.zeros(64, 1, 128), None, zeros, sequence_list([64]), 1)
    weights = torch.exp(decay * torch.arange(63, -1, -1, dtype=torch.float64))
    off = off + 2.0 ** -62 * (k.double().abs() * weights[:, None, None]).max() * v.double().abs().sum(0)[0]
    close(state, new, off, "state_out")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dk", [64, 128])
def test_rows_whose_weights_differ_by_2_to_the_36(dtype, dk):
    """Row 0 meets one v; behind a decay of +25 the same v and its negative meet weights 2^36 times as large, which cancel."""
    def edit(q, k, v, g, st):
        st.zero_()
        k[1] = k[0]
        v[1], v[2:32] = -v[0], 0.0
        g.zero_()
        g[32] = 25.0
    run(dtype, [40], 2, 1, dk, 64, edit=edit)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 200)])
def test_columns_of_a_state_that_differ_by_2_to_the_100(dtype, dk, dv):
    """Element (0, 0) of each state is 1e30 and alone in its column; q does not meet it."""
    def edit(q, k, v, g, st):
        q[:, :, 0], v[:, :, 0] = 0.0, 0.0
        st[:, :, :, 0] = 0.0
        st[:, :, 0, 0] = 1e30
    run(dtype, [100], 2, 2, dk, dv, edit=edit)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dk", [64, 128])
def test_decays_that_grow_as_far_as_they_may(dtype, dk):
    """e^69 in a chunk, met by the largest k of fp16: weighted ones of 2^115.  scale brings the last rows into the type's range."""
    def edit(q, k, v, g, st):
        g.fill_(1.08)
        k[3] = 65504.0
        k[20] = -65504.0
        v.mul_(2.0 ** -10)
        st.mul_(2.0 ** -10)
    run(dtype, [64], 2, 1, dk, 64, edit=edit, scale=2.0 ** -118)
