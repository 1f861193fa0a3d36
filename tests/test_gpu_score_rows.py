"""Long rows on CTAs of 128 threads (from four rows an SM on) against 64 bits.

Tolerances, derived like those of test_gpu_score.py, with the terms that a thread of such a CTA adds up: at most ceil(vocab / 128) + 8 one
after the other, and the trees above it at most 17 - 2."""
import pytest
import torch

from paper_2505_07004_b200 import api as libgq
from test_gpu_score import DT, U, close, make, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    return torch.device("cuda:0")


@pytest.mark.parametrize("dtype,n,vocab,top,pad", [("bf16", 1200, 50001, 20, 0), ("fp16", 1200, 50001, 32, 7), ("fp32", 1300, 40000, 20, 0),
                                                   ("bf16", 2400, 8192 * 3 + 5, 0, 3), ("fp32", 640, 33333, 5, 1), ("fp16", 1200, 129, 32, 0)])
def test_long_rows_on_narrow_ctas(dev, dtype, n, vocab, top, pad):
    sms = torch.cuda.get_device_properties(dev).multi_processor_count
    assert n >= 4 * sms
    x, t, _ = make(dev, n, vocab, DT[dtype], seed=vocab, pad=pad)
    t[::7] = -100
    logp, entropy, stats, top_logp, top_ids = libgq.gq_token_logprobs(x, t, top=top)
    libgq.gq_check()
    tol = (vocab / 128 + 69) * U
    for r0 in range(0, n, 400):                           # 64-bit copies of a part of the rows at a time
        s = slice(r0, min(n, r0 + 400))
        m, L, logp_w, ent_w, tl_w, ti_w = reference(x[s], t[s], top)
        assert torch.equal(stats[s, 0].double(), m)
        close(stats[s, 1], L, tol + 2 * U * L.abs())
        close(logp[s], logp_w, tol + 2 * U * (logp_w.abs() + L.abs()))
        close(entropy[s], ent_w, tol * (1 + 2 * (ent_w + L)) + 2 * U * ent_w)
        if top:
            assert torch.equal(top_ids[s].long(), ti_w)
            close(top_logp[s], tl_w, tol + 2 * U * (tl_w.abs() + L[:, None].abs()))
