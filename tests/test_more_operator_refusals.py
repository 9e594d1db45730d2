"""What the gated delta rule, the norm and the 8-bit products refuse, before anything is launched: no GPU needed."""
import ctypes

import pytest
import torch

from paper_2608_20725_b200 import binding

OK, INVALID, NULL, MISALIGNED, UNSUPPORTED = 0, 1, 2, 3, 5
A = 1 << 20                # an address, aligned; nothing is read from it
MOST = 2 ** 31 - 4096


def delta(q=A, k=A, v=A, g=A, beta=A, o=A, state=None, state_out=None, cu=None, slots_at=None, dtype=binding.BF16, **sizes):
    s = dict(tokens=8, sequences=2, slots=0, max_len=0, heads=4, qk_heads=2, dk=64, dv=64, normalize=1, scale=1.0, q_stride=128, k_stride=128,
             v_stride=256, o_stride=256, decay_stride=4, beta_stride=4)
    s.update(sizes)
    seqs = binding.Sequences(cu, slots_at, None)
    return binding.lib().im2win_gated_delta_rule(q, k, v, g, beta, o, state, state_out, ctypes.byref(seqs), ctypes.byref(binding.DeltaShape(**s)),
                                                 dtype, None)


@pytest.mark.parametrize("status,call", [
    (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(g=None)), (NULL, dict(beta=None)), (NULL, dict(o=None)),
    (INVALID, dict(heads=0)), (INVALID, dict(qk_heads=0)), (INVALID, dict(qk_heads=3)), (INVALID, dict(dk=0)), (INVALID, dict(dv=0)),
    (INVALID, dict(tokens=-1)), (INVALID, dict(tokens=9)), (INVALID, dict(sequences=0)), (INVALID, dict(max_len=-1)), (INVALID, dict(dtype=3)),
    (INVALID, dict(q_stride=127)), (INVALID, dict(k_stride=127)), (INVALID, dict(v_stride=255)), (INVALID, dict(o_stride=255)),
    (INVALID, dict(decay_stride=3)), (INVALID, dict(beta_stride=3)), (INVALID, dict(normalize=2)), (INVALID, dict(normalize=-1)),
    (INVALID, dict(state=A)), (INVALID, dict(state_out=A, slots=1)), (INVALID, dict(slots_at=A)),
    (MISALIGNED, dict(q=A + 1)), (MISALIGNED, dict(o=A + 1)), (MISALIGNED, dict(g=A + 2)), (MISALIGNED, dict(beta=A + 2)),
    (MISALIGNED, dict(state=A + 4, slots=2)), (MISALIGNED, dict(state_out=A + 8, slots=2)), (MISALIGNED, dict(cu=A + 1)),
    (UNSUPPORTED, dict(dk=257, q_stride=1024, k_stride=1024)), (UNSUPPORTED, dict(dv=2 ** 30, v_stride=2 ** 33, o_stride=2 ** 33)),
    (UNSUPPORTED, dict(tokens=MOST + 2, cu=A)), (UNSUPPORTED, dict(tokens=0, sequences=MOST + 1, cu=A)),
], ids=str)
def test_delta_rule_refuses(status, call):
    assert delta(**call) == status


def test_delta_rule_kernel_names():
    assert binding.im2win_gated_delta_rule_kernel_name(binding.make_delta_shape(8, 2, 4, 3, 64, 64), binding.BF16) == "none"
    assert binding.im2win_gated_delta_rule_kernel_name(binding.make_delta_shape(8, 2, 4, 2, 257, 64), binding.BF16) == "none"
    for code in (binding.F32, binding.F16, binding.BF16):
        assert binding.im2win_gated_delta_rule_kernel_name(binding.make_delta_shape(8, 8, 4, 2, 64, 64, 1), code) == "tokens"


def norm(x=A, residual=A, weight=A, out=A, y=A, scales=None, dtype=binding.BF16, **sizes):
    s = dict(rows=4, channels=64, eps=1e-6, x_stride=64, residual_stride=64, residual_out_stride=64, y_stride=64)
    s.update(sizes)
    return binding.lib().im2win_rms_norm(x, residual, weight, out, y, scales, ctypes.byref(binding.NormShape(**s)), dtype, None)


@pytest.mark.parametrize("status,call", [
    (NULL, dict(x=None)), (NULL, dict(y=None)), (INVALID, dict(rows=-1)), (INVALID, dict(channels=0)), (INVALID, dict(eps=-1.0)),
    (INVALID, dict(eps=float("nan"))), (INVALID, dict(x_stride=63)), (INVALID, dict(residual_stride=63)), (INVALID, dict(residual_out_stride=63)),
    (INVALID, dict(y_stride=63)), (INVALID, dict(residual=None)), (INVALID, dict(dtype=3)), (MISALIGNED, dict(x=A + 1)),
    (MISALIGNED, dict(residual=A + 1)), (MISALIGNED, dict(weight=A + 1)), (MISALIGNED, dict(out=A + 1)), (MISALIGNED, dict(y=A + 1)),
    (MISALIGNED, dict(scales=A + 2)), (UNSUPPORTED, dict(rows=MOST + 1)), (OK, dict(rows=0)), (OK, dict(rows=0, x=None, y=None)),
    (OK, dict(rows=0, scales=A, y=A + 1)),
], ids=str)
def test_norm_refuses(status, call):
    assert norm(**call) == status


def matmul(x=A, x_scales=A, weight=A, scales=A, bias=None, y=A, dtype=binding.BF16, **sizes):
    s = dict(M=4, N=64, K=256, x_stride=256, y_stride=64)
    s.update(sizes)
    return binding.lib().im2win_matmul_int8(x, x_scales, weight, scales, bias, y, ctypes.byref(binding.Int8Shape(**s)), dtype, None)


@pytest.mark.parametrize("status,call", [
    (NULL, dict(x=None)), (NULL, dict(x_scales=None)), (NULL, dict(weight=None)), (NULL, dict(scales=None)), (NULL, dict(y=None)),
    (INVALID, dict(M=-1)), (INVALID, dict(N=0)), (INVALID, dict(K=0)), (INVALID, dict(x_stride=255)), (INVALID, dict(y_stride=63)),
    (INVALID, dict(dtype=3)), (UNSUPPORTED, dict(K=131072, x_stride=131072)), (UNSUPPORTED, dict(M=MOST + 1)), (MISALIGNED, dict(y=A + 1)),
    (MISALIGNED, dict(scales=A + 2)), (MISALIGNED, dict(x_scales=A + 2)), (MISALIGNED, dict(bias=A + 1)), (OK, dict(M=0, x=None, y=None)),
], ids=str)
def test_matmul_refuses(status, call):
    assert matmul(**call) == status


def test_matmul_kernel_names():
    assert binding.im2win_matmul_int8_kernel_name(0, 0, 1, binding.F32) == "none"
    assert binding.im2win_matmul_int8_kernel_name(4, 64, 131072, binding.F32) == "none"
    assert binding.im2win_matmul_int8_kernel_name(4, 64, 33, binding.F32) == "registers"


def test_missing_shapes():
    L = binding.lib()
    assert L.im2win_gated_delta_rule(A, A, A, A, A, A, None, None, None, None, 0, None) == NULL
    assert L.im2win_rms_norm(A, None, A, None, A, None, None, 0, None) == NULL
    assert L.im2win_matmul_int8(A, A, A, A, None, A, None, 0, None) == NULL


def test_structures_and_their_bytes_agree():
    assert bytes(binding.DeltaShape(*range(1, 10), 0.5, *range(11, 17))) == binding._pack_delta(*range(1, 10), 0.5, *range(11, 17))
    assert bytes(binding.NormShape(1, 2, 0.5, 3, 4, 5, 6)) == binding._pack_norm(1, 2, 0.5, 3, 4, 5, 6)
    assert bytes(binding.Int8Shape(1, 2, 3, 4, 5)) == binding._pack_int8(1, 2, 3, 4, 5)


def test_binding_refuses_what_does_not_fit():
    x = torch.zeros(4, 2, 8)
    with pytest.raises(ValueError, match="CUDA device"):
        binding.im2win_gated_delta_rule(x, x, x, torch.zeros(4, 2), torch.zeros(4, 2), x)
    with pytest.raises(ValueError, match="CUDA device"):
        binding.im2win_rms_norm(x[0], None, x[0])
    with pytest.raises(ValueError, match="CUDA device"):
        binding.im2win_matmul_int8(x[0].to(torch.int8), torch.zeros(2), torch.zeros(8, 8, dtype=torch.int8), torch.zeros(8), torch.zeros(2, 8))
    with pytest.raises(TypeError):
        binding.im2win_rms_norm(x[0].double(), None, x[0])
    pick = binding._by_token_or_head
    assert pick(torch.zeros(4, 2), 2, (4, 2), 4, "beta") == 2 and pick(torch.zeros(2), 2, (4, 2), 4, "beta") == 0
    assert pick(torch.zeros(2).expand(4, 2), 2, (4, 2), 4, "beta") == 0 and pick(torch.zeros(4, 6)[:, :2], 2, (4, 2), 4, "beta") == 6
    for bad in (torch.zeros(4, 3), torch.zeros(4, 2).double(), torch.zeros(2, 4).T):
        with pytest.raises(ValueError):
            pick(bad, 2, (4, 2), 4, "beta")
