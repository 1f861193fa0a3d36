"""Refusals of the token scores (gq_token_logprobs, gq_token_logprobs_grad): found on the host, nothing is launched."""
import ctypes

import pytest
import torch

from paper_2505_07004_b200 import api as libgq
from paper_2505_07004_b200 import build as gq_build

INVALID, ALIGN, SHAPE = -1, -2, -3
REFUSED = (INVALID, ALIGN, SHAPE, -4)


@pytest.fixture(scope="module")
def L():
    gq_build.build_libgq()
    return libgq.lib()


@pytest.fixture(scope="module")
def base():
    buf = (ctypes.c_uint8 * (1 << 16))()
    base.keep = buf
    return (ctypes.addressof(buf) + 127) // 128 * 128


def test_scores(L, base):
    x, t, lp, en, st, tl, ti = (base + 4096 * i for i in range(7))

    def call(x=x, dtype=0, n=3, vocab=40, ld=40, t=t, top=2, lp=lp, en=en, st=st, tl=tl, ti=ti):
        return L.gq_token_logprobs(x, dtype, n, vocab, ld, t, top, lp, en, st, tl, ti, None)
    assert call(dtype=3) == INVALID and call(dtype=-1) == INVALID
    assert call(n=-1) == INVALID and call(vocab=0) == INVALID and call(ld=39) == INVALID
    assert call(vocab=(1 << 30) + 1, ld=1 << 31) == SHAPE and call(n=1 << 28) == SHAPE
    assert call(top=-1) == INVALID and call(top=41) == INVALID and call(top=33) == SHAPE
    assert call(x=None) == INVALID and call(en=None) == INVALID and call(st=None) == INVALID
    assert call(t=None) == INVALID and call(lp=None) == INVALID              # one without the other
    assert call(tl=None) == INVALID and call(ti=None) == INVALID
    assert call(x=x + 1) == ALIGN and call(dtype=2, x=x + 2) == ALIGN and call(t=t + 4) == ALIGN and call(lp=lp + 2) == ALIGN
    assert call(st=st + 1) == ALIGN and call(ti=ti + 2) == ALIGN
    assert call(lp=x + 4) == INVALID and call(en=lp + 8) == INVALID and call(st=t) == INVALID and call(tl=ti + 4) == INVALID
    assert call(x=None, n=0, t=None, lp=None) == 0                           # nothing to do: pointers are not looked at
    # what is allowed gets as far as the device (none here)
    for ok in (call(), call(x=x + 2), call(t=None, lp=None), call(top=0, tl=None, ti=None), call(top=32), call(vocab=1, ld=1, top=1)):
        assert ok not in REFUSED


def test_gradient(L, base):
    x, t, st, en, dl, de, dx = (base + 4096 * i for i in range(7))

    def call(x=x, dtype=0, n=3, vocab=40, ld=40, t=t, st=st, en=en, dl=dl, de=de, dx=dx, ld_d=40):
        return L.gq_token_logprobs_grad(x, dtype, n, vocab, ld, t, st, en, dl, de, dx, ld_d, None)
    assert call(dtype=3) == INVALID and call(n=-1) == INVALID and call(vocab=0) == INVALID and call(ld=39) == INVALID
    assert call(ld_d=39) == INVALID and call(n=1 << 28) == SHAPE
    assert call(x=None) == INVALID and call(st=None) == INVALID and call(dx=None) == INVALID
    assert call(t=None) == INVALID and call(dl=None) == INVALID              # one without the other
    assert call(t=None, dl=None, de=None) == INVALID                         # no gradient at all
    assert call(en=None) == INVALID                                          # an entropy gradient needs the entropy
    assert call(dx=dx + 1) == ALIGN and call(dtype=2, dx=dx + 2) == ALIGN and call(de=de + 2) == ALIGN and call(t=t + 4) == ALIGN
    assert call(dx=x) == INVALID and call(dx=st - 16) == INVALID
    assert call(x=None, n=0, t=None, dl=None, de=None, dx=None) == 0
    for ok in (call(), call(de=None, en=None), call(t=None, dl=None), call(dx=dx + 2)):
        assert ok not in REFUSED


def test_binding_refuses_host_tensors_and_shapes():
    with pytest.raises(ValueError, match="CUDA tensor"):
        libgq.gq_token_logprobs(torch.zeros(2, 8))
    with pytest.raises(ValueError, match="CUDA tensor"):
        libgq.gq_token_logprobs_grad(torch.zeros(2, 8), None, torch.zeros(2, 2))


def test_timing_arrays_keep_their_size(L):
    """A caller compiled for 14 kernels gets 14 entries; the new ones have a call that is told how many there are."""
    ms, n = (ctypes.c_double * 18)(*[-1.0] * 18), (ctypes.c_uint64 * 18)()
    assert L.gq_kernel_timing_read(ms, n) == 0 and ms[13] == 0.0 and ms[14] == -1.0
    assert len(libgq.KERNEL_NAMES) == 17
    assert L.gq_kernel_timing_read_all(ms, n, 17) == 0 and ms[16] == 0.0 and ms[17] == -1.0
    assert L.gq_kernel_timing_read_all(ms, n, 18) == INVALID and L.gq_kernel_timing_read_all(ms, n, 0) == INVALID
    assert L.gq_kernel_timing_read_all(None, n, 17) == INVALID
