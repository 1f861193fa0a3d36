"""A stream handle that is not a torch.cuda.Stream, as the library's other calls take it."""
import types

import pytest
import torch

from paper_2505_07004_b200 import api as libgq

pytestmark = pytest.mark.gpu


def test_calls_on_a_plain_stream_handle():
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(1)
    Q = torch.randint(0, 16, (40, 72), generator=gen, device=dev, dtype=torch.uint8)
    codebook = torch.randn(40, 16, generator=gen, device=dev)
    X = torch.randn(9, 72, generator=gen, device=dev).bfloat16()
    t = torch.arange(9, device=dev)
    side = torch.cuda.Stream()

    def chain(stream):
        codes, table = libgq.gq_linear_pack(Q, codebook, stream=stream)
        Y = libgq.gq_linear(X, codes, table, 16, stream=stream)
        ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(9, 72, 40), dev)
        grads = libgq.gq_linear_grad(Y, X, codes, table, 16, ws, stream=stream)
        logp, entropy, stats, top_logp, top_ids = libgq.gq_token_logprobs(Y, t, top=3, stream=stream)
        d = libgq.gq_token_logprobs_grad(Y, t, stats, entropy, logp, logp, stream=stream)
        return [Y, *grads, logp, entropy, stats, top_logp, top_ids, d, ws]
    want = chain(None)
    torch.cuda.synchronize()
    for handle in (side, types.SimpleNamespace(device=dev, cuda_stream=side.cuda_stream), types.SimpleNamespace(cuda_stream=side.cuda_stream)):
        got = chain(handle)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[:-1], got[:-1]))
    libgq.gq_check()
