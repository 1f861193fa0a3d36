"""Sizes that the products' kernels do not index are refused before anything is launched.  (Made-up addresses, far apart; nothing reads them.)"""
import pytest

from paper_2505_07004_b200 import api as libgq
from paper_2505_07004_b200 import build as gq_build

SHAPE = -3
FAR = 1 << 52


@pytest.fixture(scope="module")
def L():
    gq_build.build_libgq()
    return libgq.lib()


def test_forward(L):
    n, d = 1 << 28, 1 << 20
    assert L.gq_linear(FAR, 0, n, 8, 8, 2 * FAR, 3 * FAR, 16, d, None, 0, None, 0, 4 * FAR, d, None, 0, None) == SHAPE


@pytest.mark.parametrize("dx,dt", [(True, False), (False, True), (True, True)])
def test_gradient(L, dx, dt):
    n, d = 1 << 28, 1 << 20
    d_out = d if dt else 8
    ws = L.gq_linear_grad_workspace_bytes(n, d, d_out)
    assert L.gq_linear_grad(FAR, 0, n, d_out, d_out, 2 * FAR, d_out, 2, 3 * FAR, d, d, 4 * FAR, 5 * FAR, 16, 6 * FAR, d_out, 7 * FAR if dx else None, d,
                            8 * FAR if dt else None, None, 9 * FAR, ws, None) == SHAPE
