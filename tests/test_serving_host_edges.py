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


def test_arguments_that_are_no_tensors_are_refused_as_such(S):
    p, cu = torch.zeros(2, 2, 64).bfloat16(), torch.tensor([0, 2], dtype=torch.int32)
    codes, params = torch.zeros(2, 1, 16, 32, dtype=torch.uint8), torch.zeros(2, 1, 16, 2, 2, dtype=torch.bfloat16)
    for call in (lambda: S.attention_prompt(None, p, p, cu), lambda: S.attention_prompt(p, 3, p, cu), lambda: S.attention_prompt(p, p, p, [0, 2]),
                 lambda: S.KV4Cache(None, params, codes, params), lambda: S.KV4Cache(codes, params, codes, 1), lambda: S.query_status(0)):
        with pytest.raises(TypeError, match="torch.Tensor"):
            call()
    for word in (torch.zeros(1, dtype=torch.int32), torch.zeros(1), torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(ValueError, match="status word"):
            S.query_status(word)
