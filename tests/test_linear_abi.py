"""Refusals and sizes of the products with quantised weights: found on the host, nothing is launched."""
import ctypes

import pytest
import torch

from paper_2505_07004_b200 import api as libgq
from paper_2505_07004_b200 import build as gq_build

INVALID, ALIGN, SHAPE, WS = -1, -2, -3, -4
REFUSED = (INVALID, ALIGN, SHAPE, WS)
SLOT = 1 << 14


@pytest.fixture(scope="module")
def L():
    gq_build.build_libgq()
    return libgq.lib()


@pytest.fixture(scope="module")
def mem():
    buf = (ctypes.c_uint8 * (SLOT * 20))()
    mem.keep = buf
    at = (ctypes.addressof(buf) + 1023) // 1024 * 1024
    return [at + SLOT * i for i in range(18)]


def test_sizes(L):
    assert L.gq_linear_codes_bytes(64, 24) == 24 * 32
    assert L.gq_linear_codes_bytes(72, 24) == 24 * 48                   # rows padded to whole 16 bytes
    assert L.gq_linear_codes_bytes(68, 24) == 0 and L.gq_linear_codes_bytes(64, 20) == 0 and L.gq_linear_codes_bytes(0, 8) == 0
    assert L.gq_linear_codes_bytes((1 << 20) + 8, 8) == 0
    # one part of sums for both halves of a feature tile (256 channels are one tile), one row of column sums for 16 tokens
    assert L.gq_linear_grad_workspace_bytes(16, 256, 256) == 2 * 256 * 64 + 1024
    assert L.gq_linear_grad_workspace_bytes(17, 256, 264) == 2 * 264 * 64 + (2 * 264 * 4 + 1023) // 1024 * 1024
    assert L.gq_linear_grad_workspace_bytes(-1, 256, 256) == 0 and L.gq_linear_grad_workspace_bytes(1, 255, 256) == 0


def test_pack(L, mem):
    q, cb, codes, table = mem[:4]

    def call(q=q, cb=cb, m=16, d_in=72, d_out=16, dtype=0, codes=codes, table=table):
        return L.gq_linear_pack(q, cb, m, d_in, d_out, dtype, codes, table, None)
    assert call(dtype=2) == INVALID and call(m=0) == INVALID and call(m=17) == SHAPE
    assert call(d_in=70) == SHAPE and call(d_out=12) == SHAPE and call(d_in=0) == INVALID
    assert call(q=None) == INVALID and call(codes=None) == INVALID and call(table=None) == INVALID and call(cb=None) == INVALID
    assert call(codes=codes + 8) == ALIGN and call(table=table + 2) == ALIGN and call(cb=cb + 2) == ALIGN
    assert call(codes=q) == INVALID and call(table=codes + 16) == INVALID
    assert call() not in REFUSED and call(q=q + 1) not in REFUSED


def test_linear(L, mem):
    x, codes, table, bias, res, y, z = mem[:7]

    def call(x=x, dtype=0, n=3, d_in=72, ld_x=72, codes=codes, table=table, m=16, d_out=24, bias=bias, act=2, res=res, ld_r=24, y=y, ld_y=24,
             z=z, ld_z=24):
        return L.gq_linear(x, dtype, n, d_in, ld_x, codes, table, m, d_out, bias, act, res, ld_r, y, ld_y, z, ld_z, None)
    assert call(dtype=2) == INVALID and call(dtype=3) == INVALID and call(n=-1) == INVALID and call(m=0) == INVALID
    assert call(m=17) == SHAPE and call(d_in=71) == SHAPE and call(d_out=20) == SHAPE and call(n=(1 << 28) + 1) == SHAPE
    assert call(act=-1) == INVALID and call(act=4) == INVALID
    assert call(ld_x=64) == INVALID and call(ld_y=16) == INVALID and call(ld_r=16) == INVALID and call(ld_z=16) == INVALID
    assert call(ld_x=76) == ALIGN and call(ld_y=28) == ALIGN and call(ld_r=28) == ALIGN and call(ld_z=28) == ALIGN
    assert call(x=x + 8) == ALIGN and call(y=y + 2) == ALIGN and call(codes=codes + 8) == ALIGN and call(table=table + 8) == ALIGN
    assert call(bias=bias + 1) == ALIGN and call(res=res + 4) == ALIGN and call(z=z + 8) == ALIGN
    assert call(x=None) == INVALID and call(codes=None) == INVALID and call(table=None) == INVALID and call(y=None) == INVALID
    assert call(y=x) == INVALID and call(y=res) == INVALID and call(z=y + 16) == INVALID and call(y=codes) == INVALID and call(z=table) == INVALID
    assert call(n=0, x=None, y=None, codes=None) == 0
    for ok in (call(), call(bias=None, res=None, z=None, ld_r=0, ld_z=0), call(n=8), call(n=9), call(m=1), call(res=x, ld_r=72)):
        assert ok not in REFUSED


def test_gradient(L, mem):
    dy, z, x, codes, table, dz, dx, dt, db, ws = mem[:10]
    need = L.gq_linear_grad_workspace_bytes(3, 72, 24)

    def call(dy=dy, dtype=0, n=3, d_out=24, ld_dy=24, z=z, ld_z=24, act=2, x=x, d_in=72, ld_x=72, codes=codes, table=table, m=16, dz=dz, ld_dz=24,
             dx=dx, ld_dx=72, dt=dt, db=db, ws=ws, ws_bytes=need):
        return L.gq_linear_grad(dy, dtype, n, d_out, ld_dy, z, ld_z, act, x, d_in, ld_x, codes, table, m, dz, ld_dz, dx, ld_dx, dt, db, ws, ws_bytes, None)
    assert call(dtype=2) == INVALID and call(n=-1) == INVALID and call(m=17) == SHAPE and call(d_in=70) == SHAPE and call(act=4) == INVALID
    assert call(z=None) == INVALID and call(dz=None) == INVALID            # an activation needs both
    assert call(act=0) == INVALID and call(act=0, z=None) == INVALID       # without one they are not given
    assert call(dy=None) == INVALID and call(codes=None) == INVALID and call(x=None) == INVALID
    assert call(table=None) == INVALID
    assert call(ld_dy=16) == INVALID and call(ld_dx=64) == INVALID and call(ld_x=64) == INVALID and call(ld_dz=28) == ALIGN
    assert call(dx=dx + 8) == ALIGN and call(dt=dt + 2) == ALIGN and call(db=db + 1) == ALIGN and call(ws=ws + 16) == ALIGN
    assert call(ws=None) == WS and call(ws_bytes=need - 1) == WS
    assert call(dz=dy) == INVALID and call(dx=x) == INVALID and call(dt=ws) == INVALID and call(db=dt + 8) == INVALID and call(dx=codes) == INVALID
    for ok in (call(), call(act=0, z=None, dz=None, ld_z=0, ld_dz=0), call(dt=None, db=None, ws=None, ws_bytes=0, x=None), call(dx=None),
               call(dx=None, dt=None, codes=None, table=None, x=None)):
        assert ok not in REFUSED


def test_binding_refuses_host_tensors():
    with pytest.raises(ValueError, match="CUDA tensor"):
        libgq.gq_linear_pack(torch.zeros(8, 8, dtype=torch.uint8), torch.zeros(8, 4))
    with pytest.raises(ValueError, match="CUDA tensor"):
        libgq.gq_linear(torch.zeros(1, 8, dtype=torch.bfloat16), torch.zeros(8, 16, dtype=torch.uint8), torch.zeros(8, 16, dtype=torch.bfloat16), 16)
