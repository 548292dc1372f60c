"""Sizes at and beyond what the paged calls take."""

import pytest
import torch

import paged_oracle as O
from test_gpu_paged_cache import assert_rotated, context, plan_of, random

pytestmark = pytest.mark.gpu

MOST_HEADS = 65535 * 8 * 4            # blocks of a grid's second dimension, groups of rows per warp, rows of a group


def test_rope_of_very_many_heads():
    """Above the most heads that a launch covers the call is refused as such, and nothing is launched."""
    B, sk = context(1, 1, 1)
    plan, freq, amp = plan_of(B, (128, False, None))
    x, pos = random(1, 1, 128), torch.tensor([3], dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 7.0)
    for heads in (MOST_HEADS + 1, 2 ** 31 - 1):
        with pytest.raises(B.SagekvError) as e:
            B.sagekv_rope(sk.ctx, plan, x, 1, heads, pos, out)
        assert e.value.code == B.ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert torch.all(out == 7) and sk.status() == 0
    x = random(1, MOST_HEADS, 128)
    out = sk.rope(x, pos, plan)
    for part in (slice(0, 5000), slice(MOST_HEADS // 2, MOST_HEADS // 2 + 5000), slice(MOST_HEADS - 5000, MOST_HEADS)):
        assert_rotated(out[:, part], x[:, part], pos, freq, False, amp)
    for few in (262140, 262141):
        assert torch.equal(sk.rope(x[:, :few], pos, plan), out[:, :few])
    sk.close()
