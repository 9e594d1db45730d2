"""What the operators on token sequences refuse, before anything is launched: no GPU needed."""
import ctypes

import pytest
import torch

from paper_2608_20725_b200 import binding

OK, INVALID, NULL, MISALIGNED, SMALL, UNSUPPORTED = 0, 1, 2, 3, 4, 5
A = 1 << 20                # an address, aligned; nothing is read from it


def conv(x=A, weight=A, bias=None, y=A, state=None, state_out=None, cu=None, slots=None, dtype=binding.BF16, **sizes):
    s = dict(tokens=8, sequences=2, slots=0, channels=64, taps=4, silu=1, x_stride=64, y_stride=64)
    s.update(sizes)
    seqs = binding.Sequences(cu, slots, None)
    return binding.lib().im2win_causal_conv1d(x, weight, bias, y, state, state_out, ctypes.byref(seqs),
                                              ctypes.byref(binding.Conv1dShape(**s)), dtype, None)


@pytest.mark.parametrize("status,call", [
    (NULL, dict(x=None)), (NULL, dict(y=None)), (NULL, dict(weight=None)),
    (INVALID, dict(channels=0)), (INVALID, dict(taps=0)), (INVALID, dict(taps=9)), (INVALID, dict(silu=2)), (INVALID, dict(tokens=-2)),
    (INVALID, dict(sequences=0)), (INVALID, dict(tokens=9)), (INVALID, dict(x_stride=63)), (INVALID, dict(y_stride=0)),
    (INVALID, dict(dtype=3)), (INVALID, dict(dtype=-1)), (INVALID, dict(slots=-1)),
    (INVALID, dict(state=A)), (INVALID, dict(state_out=A, slots=1)), (INVALID, dict(slots_at=A)),
    (MISALIGNED, dict(x=A + 1)), (MISALIGNED, dict(y=A + 1)), (MISALIGNED, dict(weight=A + 1)), (MISALIGNED, dict(bias=A + 2)),
    (MISALIGNED, dict(state=A + 1, slots=2)), (MISALIGNED, dict(cu=A + 2)), (MISALIGNED, dict(slots_at=A + 2, slots=2)),
    (MISALIGNED, dict(x=A + 2, dtype=binding.F32)), (UNSUPPORTED, dict(channels=2 ** 31 - 1, x_stride=2 ** 31, y_stride=2 ** 31)),
], ids=str)
def test_conv_refuses(status, call):
    call = dict(call)
    lib_slots = call.pop("slots_at", None)
    pool = call.pop("slots", None)
    if pool is not None:
        s = dict(tokens=8, sequences=2, slots=pool, channels=64, taps=4, silu=1, x_stride=64, y_stride=64)
        seqs = binding.Sequences(call.get("cu"), lib_slots, None)
        got = binding.lib().im2win_causal_conv1d(A, A, None, A, call.get("state"), call.get("state_out"), ctypes.byref(seqs),
                                                 ctypes.byref(binding.Conv1dShape(**s)), binding.BF16, None)
    else:
        got = conv(slots=lib_slots, **call)
    assert got == status


def test_conv_refuses_a_missing_shape():
    assert binding.lib().im2win_causal_conv1d(A, A, None, A, None, None, None, None, 0, None) == NULL


def test_bf16_is_no_type_of_the_layers():
    with pytest.raises(binding.Im2winError) as e:
        binding.im2win_workspace_size(dict(N=1, C=16, H=14, W=14, Co=16, Kh=3, Kw=3, stride=1, pad=1), binding.BF16)
    assert e.value.code == INVALID


def test_binding_refuses_tensors_of_the_host_and_other_types():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="CUDA device"):
        binding.im2win_causal_conv1d(x, torch.zeros(8, 4), torch.zeros(4, 8))
    with pytest.raises(TypeError):
        binding.im2win_causal_conv1d(x.double(), torch.zeros(8, 4), torch.zeros(4, 8))


def test_binding_row_strides():
    r = binding._row_stride
    assert r(torch.zeros(5, 12)[:, 2:9], 1, "x") == 12
    assert r(torch.zeros(1, 12)[:, 2:9], 1, "x") == 7
    assert r(torch.zeros(3, 5, 12)[:, :, 2:9], 1, "x") == 12
    assert r(torch.zeros(3, 5, 12)[:, :1], 1, "x") == 60
    assert r(torch.zeros(3, 5, 12)[:1], 1, "x") == 12
    assert r(torch.zeros(4, 3, 8), 2, "q") == 24
    assert r(torch.zeros(4, 60)[:, :24].unflatten(1, (3, 8)), 2, "q") == 60
    assert r(torch.zeros(6, 1), 1, "x") == 1
    for bad, inner in ((torch.zeros(5, 12).T, 1), (torch.zeros(3, 5, 12)[:, :2], 1), (torch.zeros(4, 3, 8).transpose(1, 2), 2),
                       (torch.zeros(4, 3, 9)[:, :, :8], 2), (torch.zeros(5, 3, 12).transpose(0, 1), 1)):
        with pytest.raises(ValueError):
            r(bad, inner, "x")


def meta(*shape, dtype=torch.int32):
    return torch.zeros(*shape, dtype=dtype)


def test_binding_refuses_sequences_that_do_not_fit():
    take = binding._take_sequences
    assert take((6,), None, None, None, None, None)[:3] == (6, 6, 0)
    assert take((3, 4), None, None, None, None, None)[:3] == (12, 3, 0)
    assert take((9,), meta(4), None, None, torch.zeros(3, 2), None)[:3] == (9, 3, 3)
    pool = torch.zeros(3, 2)
    for args in (((3, 4), meta(4), None, None, None, None), ((9,), meta(4, dtype=torch.int64), None, None, None, None),
                 ((9,), meta(1), None, None, None, None), ((0,), None, None, None, None, None), ((6,), None, None, None, pool, None),
                 ((3,), None, None, None, pool, torch.zeros(4, 2)), ((3,), None, meta(2), None, pool, pool),
                 ((3,), None, meta(3, dtype=torch.int64), None, pool, pool), ((3,), None, None, meta(3), pool, pool),
                 ((3,), None, None, meta(2, dtype=torch.bool), pool, pool), ((2,), None, None, None, torch.zeros(2, 3).T, None),
                 ((1,), None, None, None, torch.zeros(0, 2), None)):
        with pytest.raises(ValueError):
            take(*args)


def attention(q=A, k=A, v=A, g=A, o=A, state=None, state_out=None, cu=None, slots_at=None, workspace=A, workspace_bytes=1 << 40,
              dtype=binding.BF16, **sizes):
    s = dict(tokens=8, sequences=2, slots=0, max_len=0, heads=4, qk_heads=2, dk=64, dv=64, scale=1.0, q_stride=128, k_stride=128,
             v_stride=256, o_stride=256, decay_stride=4)
    s.update(sizes)
    seqs = binding.Sequences(cu, slots_at, None)
    return binding.lib().im2win_linear_attention(q, k, v, g, o, state, state_out, ctypes.byref(seqs), workspace, workspace_bytes,
                                                 ctypes.byref(binding.AttentionShape(**s)), dtype, None)


@pytest.mark.parametrize("status,call", [
    (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(g=None)), (NULL, dict(o=None)), (NULL, dict(workspace=None)),
    (INVALID, dict(heads=0)), (INVALID, dict(qk_heads=0)), (INVALID, dict(qk_heads=3)), (INVALID, dict(dk=0)), (INVALID, dict(dv=0)),
    (INVALID, dict(tokens=-1)), (INVALID, dict(tokens=9)), (INVALID, dict(sequences=0)), (INVALID, dict(max_len=-1)), (INVALID, dict(dtype=3)),
    (INVALID, dict(q_stride=127)), (INVALID, dict(k_stride=127)), (INVALID, dict(v_stride=255)), (INVALID, dict(o_stride=255)),
    (INVALID, dict(decay_stride=3)), (INVALID, dict(state=A)), (INVALID, dict(state_out=A, slots=1)), (INVALID, dict(slots_at=A)),
    (MISALIGNED, dict(q=A + 1)), (MISALIGNED, dict(o=A + 1)), (MISALIGNED, dict(g=A + 2)), (MISALIGNED, dict(state=A + 4, slots=2)),
    (MISALIGNED, dict(state_out=A + 8, slots=2)), (MISALIGNED, dict(workspace=A + 8)), (MISALIGNED, dict(cu=A + 1)),
    (SMALL, dict(workspace_bytes=255)),
    (UNSUPPORTED, dict(dk=257, q_stride=1024, k_stride=1024)), (UNSUPPORTED, dict(dv=2 ** 30, v_stride=2 ** 33, o_stride=2 ** 33)),
], ids=str)
def test_attention_refuses(status, call):
    assert attention(**call) == status


def test_attention_kernel_names_and_sizes():
    shape = binding.make_attention_shape(8, 2, 4, 3, 64, 64)
    assert binding.im2win_linear_attention_kernel_name(shape, binding.BF16) == "none"
    with pytest.raises(binding.Im2winError):
        binding.im2win_linear_attention_workspace_size(shape, binding.BF16)
    shape = binding.make_attention_shape(8, 8, 4, 2, 64, 64)
    for code in (binding.F32, binding.F16, binding.BF16):
        assert binding.im2win_linear_attention_kernel_name(shape, code) == "tokens"
        assert binding.im2win_linear_attention_workspace_size(shape, code) >= 256


def matvec(x=A, weight=A, scales=A, zeros=None, bias=None, y=A, dtype=binding.BF16, **sizes):
    s = dict(M=2, N=64, K=256, group=64, x_stride=256, y_stride=64)
    s.update(sizes)
    return binding.lib().im2win_matvec_int4(x, weight, scales, zeros, bias, y, ctypes.byref(binding.Int4Shape(**s)), dtype, None)


@pytest.mark.parametrize("status,call", [
    (NULL, dict(x=None)), (NULL, dict(weight=None)), (NULL, dict(scales=None)), (NULL, dict(y=None)),
    (INVALID, dict(M=0)), (INVALID, dict(N=0)), (INVALID, dict(K=0)), (INVALID, dict(group=0)), (INVALID, dict(x_stride=255)),
    (INVALID, dict(y_stride=63)), (INVALID, dict(dtype=3)), (UNSUPPORTED, dict(M=17)), (UNSUPPORTED, dict(group=16)),
    (UNSUPPORTED, dict(group=96)), (UNSUPPORTED, dict(K=2 ** 31 - 1, x_stride=2 ** 31)), (MISALIGNED, dict(x=A + 1)), (MISALIGNED, dict(y=A + 1)),
    (MISALIGNED, dict(scales=A + 1)), (MISALIGNED, dict(bias=A + 2)), (MISALIGNED, dict(x=A + 2, dtype=binding.F32)),
], ids=str)
def test_matvec_refuses(status, call):
    assert matvec(**call) == status


def test_structures_and_their_bytes_agree():
    for structure, pack, values in ((binding.Sequences, binding._pack_sequences, (A, 2 * A, 3 * A)),
                                    (binding.Conv1dShape, binding._pack_conv1d, tuple(range(1, 9))),
                                    (binding.AttentionShape, binding._pack_attention, (1, 2, 3, 4, 5, 6, 7, 8, 0.5, 9, 10, 11, 12, 13)),
                                    (binding.Int4Shape, binding._pack_int4, tuple(range(1, 7)))):
        assert bytes(structure(*values)) == pack(*values)
