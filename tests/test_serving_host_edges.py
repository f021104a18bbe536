"""What the torch side of the served attention block refuses or keeps, as far as it shows without a GPU."""
import pytest
import torch

from test_serving_host import S  # noqa: F401 (the fixture)


def test_tensors_that_require_a_gradient_are_refused(S):
    x, y = torch.zeros(2, 2, 64, requires_grad=True), torch.zeros(2, 2, 64)
    pos, inv, cu = torch.zeros(2, dtype=torch.int64), torch.ones(32), torch.tensor([0, 2], dtype=torch.int32)
    h, p = x.bfloat16(), y.bfloat16()
    calls = [lambda: S.qk_norm_rope(x, y, pos, inv), lambda: S.qk_norm_rope(y, x, pos, inv), lambda: S.attention_prompt(h, p, p, cu),
             lambda: S.attention_prompt(p, h, p, cu), lambda: S.attention_prompt(p, p, h, cu)]
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):      # and not where gradients are off
            call()
