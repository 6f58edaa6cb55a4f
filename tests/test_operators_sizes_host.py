"""Sizes that 32-bit fields of the operators' structs do not hold are refused, not cut to their low bits.  (Tensors without memory.)"""
import pytest
import torch

from paper_2505_19609_amd import binding as B

PAST = (1 << 32) + 64   # 64 in its low 32 bits


def _bf16(*shape):
    return torch.empty(shape, dtype=torch.bfloat16, device="meta")


@pytest.mark.parametrize("call", [
    lambda: B._norm_of(_bf16(1, PAST), _bf16(64), 1e-5, B.NORM_RMS),
    lambda: B.skrull_norm_workspace(_bf16(1, PAST), _bf16(64), B.NORM_RMS),
    lambda: B._norm_of(_bf16(1, 64), _bf16(64), 1e-5, 1 << 32),
    lambda: B._loss_of(_bf16(4, 64), _bf16(PAST, 64), None),
    lambda: B.skrull_loss_workspace(_bf16(4, 64), _bf16(PAST, 64), True),
    lambda: B._loss_of(_bf16(1, PAST), _bf16(100, PAST), None),
    lambda: B.skrull_rotary_init(PAST), lambda: B.skrull_rotary_init(64, PAST - 32), lambda: B.skrull_rotary_init(64, layout=1 << 32),
    lambda: B.skrull_rotary_init(64, scaling=-(1 << 32))])
def test_sizes_past_32_bits_are_refused(call):
    with pytest.raises(B.SkrullError) as e:
        call()
    assert e.value.code == B.SKRULL_EINVAL


@pytest.mark.parametrize("rows", [B.ROWS_Q, B.ROWS_K])
def test_heads_past_32_bits_are_refused(rows):
    plan = B.Plan(None, B.PlanInfo(total_q=1, total_k=1, num_q_heads=1, num_kv_heads=1, head_dim=64))
    with pytest.raises(B.SkrullError):
        B._rotary_tensor(plan.info, _bf16(1, PAST, 64), _bf16(1, PAST, 64), rows)
