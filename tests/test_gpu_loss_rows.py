"""The end loss on logits whose rows share memory."""
import pytest
import torch

from paper_2505_07004_b200.loss import end_loss, token_logprobs

pytestmark = pytest.mark.gpu


def test_rows_that_share_memory():
    """One row of logits scored against several targets, and windows over one vector: what contiguous copies give."""
    torch.manual_seed(0)
    row = torch.randn(1, 501, device="cuda:0")
    windows = torch.randn(600, device="cuda:0").as_strided((6, 501), (9, 1))
    for shared, n in ((row.expand(5, 501), 5), (windows, 6), (row.expand(5, 501)[:1], 1)):
        t = torch.arange(n, device="cuda:0") * 50
        for a, b in zip(token_logprobs(shared, t, top=3), token_logprobs(shared.contiguous(), t, top=3)):
            assert torch.equal(a, b)
    leaf = row.clone().requires_grad_()
    t = torch.arange(5, device="cuda:0")
    end_loss(leaf.expand(5, 501), t).backward()
    want = row.clone().expand(5, 501).contiguous().requires_grad_()
    end_loss(want, t).backward()
    assert torch.equal(leaf.grad, want.grad.sum(0, keepdim=True))
