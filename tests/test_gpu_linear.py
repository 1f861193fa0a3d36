"""Products with quantised weights and their gradients against 64 bits.

Tolerances, derived.  Inputs are 16-bit numbers whose products are exact in fp32.  A sum over K of them is built in steps of 16 on the
tensor cores, each of which may lose up to one unit in the last place (2^-23) of the partial sums' size, at most S = sum |a b|; the
single-token kernel adds up to 64 such sums more.  So a sum is off by at most (K / 16 + 72) 2^-23 S.  Activations: |act'| <= 1.13, and
their own fp32 evaluation (exp, erf, a quotient) is good to 2^-20 of |z|.  The result is rounded once (eps / 2 relative, half the smallest
subnormal absolute).  d_table and d_bias are fp32: their last rounding and the sums over partial results are in the same bound, with K
the number of terms."""
import pytest
import torch

from paper_2505_07004_b200 import api as libgq

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = [libgq.GQ_ACT_NONE, libgq.GQ_ACT_RELU, libgq.GQ_ACT_SILU, libgq.GQ_ACT_GELU]
STEP = 2.0 ** -23


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    return torch.device("cuda:0")


def act64(z, act):
    if act == libgq.GQ_ACT_RELU:
        return z.clamp_min(0.0)
    if act == libgq.GQ_ACT_SILU:
        return z * torch.sigmoid(z)
    if act == libgq.GQ_ACT_GELU:
        return z * torch.special.ndtr(z)
    return z


def slope64(z, act):
    if act == libgq.GQ_ACT_RELU:
        return (z > 0).double()
    if act == libgq.GQ_ACT_SILU:
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) * 0.3989422804014327


def strided(gen, dev, rows, cols, dtype, pad=0, scale=1.0):
    """[rows, cols] with `pad` columns and one row more behind it, those holding NaN."""
    buf = torch.full((rows + 1, cols + pad), float("nan"), device=dev, dtype=dtype)
    buf[:rows, :cols] = (scale * torch.randn(rows, cols, generator=gen, device=dev)).to(dtype)
    return buf[:rows, :cols]


def layer(dev, d_in, d_out, m, dtype, seed):
    gen = torch.Generator(device=dev).manual_seed(seed)
    Q = torch.randint(0, m, (d_out, d_in), generator=gen, device=dev, dtype=torch.uint8)
    codebook = 0.1 * torch.randn(d_out, m, generator=gen, device=dev)
    codes, table = libgq.gq_linear_pack(Q, codebook, dtype)
    W = codebook.to(dtype).double().gather(1, Q.long())
    return gen, Q, codebook, codes, table, W


def output(dev, rows, cols, dtype, pad):
    buf = torch.full((rows + 1, cols + pad), 99.0, device=dev, dtype=dtype)
    return buf, buf[:rows, :cols]


def untouched(buf, rows, cols):
    return bool((buf[rows:] == 99.0).all()) and bool((buf[:, cols:] == 99.0).all())


def rounded(want, tol, dtype):
    f = torch.finfo(dtype)
    return 1.001 * (tol + want.abs() * f.eps / 2) + f.smallest_normal * f.eps


def within(got, want, tol):
    bad = (got.double() - want).abs() > tol
    assert not bool((bad | ~got.isfinite()).any()), ((got.double() - want).abs() / tol).max().item()


def test_pack_layout(dev):
    gen, Q, codebook, codes, table, _ = layer(dev, 72, 24, 5, torch.float16, 1)
    Q[3, 7] = 200                                         # taken as m - 1
    codes, table = libgq.gq_linear_pack(Q, codebook, torch.float16)
    want = torch.zeros(24, 96, dtype=torch.uint8, device=dev)
    want[:, :72] = Q.clamp_max(4)
    assert torch.equal(codes, want[:, 0::2] | (want[:, 1::2] << 4))
    assert torch.equal(table[:, :5], codebook.half()) and torch.count_nonzero(table[:, 5:]) == 0


def check_forward(dev, n, d_in, d_out, m, dtype, act, bias, residual, pad, seed=0, want_z=True):
    gen, Q, codebook, codes, table, W = layer(dev, d_in, d_out, m, dtype, seed)
    X = strided(gen, dev, n, d_in, dtype, pad)
    b = (torch.randn(d_out, generator=gen, device=dev)).to(dtype) if bias else None
    r = strided(gen, dev, n, d_out, dtype, pad) if residual else None
    ybuf, Y = output(dev, n, d_out, dtype, pad)
    zbuf, Z = output(dev, n, d_out, dtype, pad) if want_z else (None, None)
    out = libgq.gq_linear(X, codes, table, m, bias=b, activation=act, residual=r, Y=Y, Z=Z)
    libgq.gq_check()
    assert out is Y and untouched(ybuf, n, d_out)
    z = X.double() @ W.t()
    S = X.double().abs() @ W.abs().t()
    if bias:
        z, S = z + b.double(), S + b.double().abs()
    tol = (d_in / 16 + 72) * STEP * S
    if want_z:
        assert untouched(zbuf, n, d_out)
        within(Z, z, rounded(z, tol, dtype))
    y = act64(z, act)
    tol = 1.13 * tol + 2.0 ** -20 * z.abs()
    if residual:
        y = y + r.double()
    tol = tol + 2.0 ** -23 * y.abs()
    within(Y, y, rounded(y, tol, dtype))
    return X, codes, table, Y


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 63, 128, 257, 520])
@pytest.mark.parametrize("d_in,d_out,m", [(8, 8, 16), (64, 264, 3), (136, 1000, 16), (1032, 248, 8)])
def test_forward_sizes(dev, dtype, n, d_in, d_out, m):
    check_forward(dev, n, d_in, d_out, m, DT[dtype], libgq.GQ_ACT_NONE, False, False, 0, seed=n)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("n", [1, 5, 40])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bias,residual,pad", [(True, False, 0), (False, True, 8), (True, True, 24)])
def test_forward_epilogue_and_strides(dev, dtype, n, act, bias, residual, pad):
    check_forward(dev, n, 200, 312, 16, DT[dtype], act, bias, residual, pad, seed=act)


@pytest.mark.parametrize("n,d_in,d_out,m", [(1, 4096, 4096, 16), (3, 11008, 512, 16), (8, 28672, 264, 8), (300, 4096, 11008, 16), (1500, 2056, 1408, 4),
                                            (600, 64, 9000, 16), (20, 28672, 256, 16), (5000, 512, 512, 16)])
def test_forward_large(dev, n, d_in, d_out, m):
    check_forward(dev, n, d_in, d_out, m, torch.bfloat16, libgq.GQ_ACT_SILU, True, True, 0, want_z=False)


@pytest.mark.parametrize("m", [1, 2, 4, 8, 9, 15, 16])
@pytest.mark.parametrize("n", [4, 100])
def test_every_level_is_found(dev, m, n):
    """One-hot activations: the outputs are the levels themselves."""
    gen, Q, codebook, codes, table, W = layer(dev, 128, 256, m, torch.bfloat16, m)
    X = torch.zeros(n, 128, dtype=torch.bfloat16, device=dev)
    at = torch.arange(n, device=dev) % 128
    X[torch.arange(n, device=dev), at] = 1.0
    Y = libgq.gq_linear(X, codes, table, m)
    libgq.gq_check()
    assert torch.equal(Y.double(), W.t()[at])


@pytest.mark.parametrize("n", [2, 70])
def test_infinite_level_zero_stays_out_of_the_padding(dev, n):
    gen, Q, codebook, codes, table, W = layer(dev, 72, 64, 16, torch.bfloat16, 3)
    Q.clamp_min_(1)
    codebook[:, 0] = float("inf")                         # the code of the padding; no weight has it
    codes, table = libgq.gq_linear_pack(Q, codebook, torch.bfloat16)
    X = torch.randn(n, 72, generator=gen, device=dev).bfloat16()
    Y = libgq.gq_linear(X, codes, table, 16)
    libgq.gq_check()
    W = codebook.bfloat16().double().gather(1, Q.long())
    z, S = X.double() @ W.t(), X.double().abs() @ W.abs().t()
    within(Y, z, rounded(z, 80 * STEP * S, torch.bfloat16))


def check_backward(dev, n, d_in, d_out, m, dtype, act, pad, seed=0):
    gen, Q, codebook, codes, table, W = layer(dev, d_in, d_out, m, dtype, seed)
    X = strided(gen, dev, n, d_in, dtype, pad)
    dY = strided(gen, dev, n, d_out, dtype, pad, 0.5)
    has = act != libgq.GQ_ACT_NONE
    Z = strided(gen, dev, n, d_out, dtype, pad, 2.0) if has else None
    zbuf, dZ = output(dev, n, d_out, dtype, pad) if has else (None, None)
    xbuf, dX = output(dev, n, d_in, dtype, pad)
    need = libgq.gq_linear_grad_workspace_bytes(n, d_in, d_out)
    ws = libgq.alloc_workspace(need, dev).fill_(0xFF)
    dZ, dX, d_table, d_bias = libgq.gq_linear_grad(dY, X, codes, table, m, ws, Z=Z, activation=act, dZ=dZ, dX=dX)
    libgq.gq_check()
    assert untouched(xbuf, n, d_in) and (not has or untouched(zbuf, n, d_out))
    if has:
        want = dY.double() * slope64(Z.double(), act)
        within(dZ, want, rounded(want, 2.0 ** -19 * dY.double().abs() * (1 + Z.double().abs()), dtype))
    else:
        assert dZ is dY
    g = dZ.double()                                       # the other gradients are those of the dZ that was returned
    want, S = g @ W, g.abs() @ W.abs()
    within(dX, want, rounded(want, (d_out / 16 + 72) * STEP * S, dtype))
    G, S = g.t() @ X.double(), g.abs().t() @ X.double().abs()
    code = Q.long()
    want = torch.zeros(d_out, m, dtype=torch.float64, device=dev).scatter_add_(1, code, G)
    S = torch.zeros(d_out, m, dtype=torch.float64, device=dev).scatter_add_(1, code, S)
    within(d_table, want, (min(n, 1024) / 16 + d_in + n / 1024 + 72) * STEP * S + 1e-37)
    within(d_bias, g.sum(0), (n / 8 + 72) * STEP * g.abs().sum(0) + 1e-37)
    return dZ, dX, d_table, d_bias


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("n", [1, 8, 65, 300, 1100])
@pytest.mark.parametrize("d_in,d_out,m", [(8, 8, 16), (264, 64, 3), (1000, 136, 16), (248, 1032, 8)])
def test_backward_sizes(dev, dtype, n, d_in, d_out, m):
    check_backward(dev, n, d_in, d_out, m, DT[dtype], libgq.GQ_ACT_NONE, 0, seed=n)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n,pad", [(3, 8), (130, 24)])
def test_backward_activations_and_strides(dev, dtype, act, n, pad):
    check_backward(dev, n, 312, 200, 16, DT[dtype], act, pad, seed=act)


@pytest.mark.parametrize("n,d_in,d_out,m", [(2048, 4096, 4096, 16), (203, 1032, 1408, 4), (4100, 512, 264, 16), (700, 256, 8200, 16), (64, 11008, 512, 8)])
def test_backward_large(dev, n, d_in, d_out, m):
    check_backward(dev, n, d_in, d_out, m, torch.bfloat16, libgq.GQ_ACT_SILU, 0)


def test_gradients_match_differences(dev):
    """The gradient of sum(C Y) along random directions of X and of the levels against central differences of a 64-bit forward pass
    over the kernel's own weights; dY = C, rounded, is what both sides use."""
    n, d_in, d_out, m, act = 40, 72, 64, 16, libgq.GQ_ACT_GELU
    gen, Q, codebook, codes, table, W = layer(dev, d_in, d_out, m, torch.float16, 5)
    X = torch.randn(n, d_in, generator=gen, device=dev).half()
    C = torch.randn(n, d_out, generator=gen, device=dev).half()
    Z = torch.empty(n, d_out, dtype=torch.float16, device=dev)
    libgq.gq_linear(X, codes, table, m, activation=act, Z=Z)
    ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(n, d_in, d_out), dev)
    _, dX, d_table, d_bias = libgq.gq_linear_grad(C, X, codes, table, m, ws, Z=Z, activation=act)
    levels, code = table[:, :m].double(), Q.long()

    def value(x, lv, b):
        return (C.double() * act64(x @ lv.gather(1, code).t() + b, act)).sum()
    zero = torch.zeros(d_out, dtype=torch.float64, device=dev)
    e = 1e-4
    for grad, move in ((dX, lambda v: (X.double() + v, levels, zero)), (d_table, lambda v: (X.double(), levels + v, zero)),
                       (d_bias, lambda v: (X.double(), levels, zero + v))):
        v = torch.randn(grad.shape, generator=gen, device=dev).double()
        numeric = (value(*move(e * v)) - value(*move(-e * v))) / (2 * e)
        # every entry of dZ (rounded from a rounded Z: slope changes by at most 0.8 |dz|) and of dX is off by a few 2^-11; in a sum of
        # N such entries with random directions 2^-9 of the root of the sum of squares is more than four standard deviations
        size = (grad.double() * v).pow(2).sum().sqrt()
        assert abs(float(numeric - (grad.double() * v).sum())) <= 2.0 ** -9 * float(size) * 4 + 1e-4


def test_runs_agree_bit_for_bit_on_streams_and_in_graphs(dev):
    n, d_in, d_out, m, act = 300, 520, 1000, 16, libgq.GQ_ACT_SILU
    gen, Q, codebook, codes, table, W = layer(dev, d_in, d_out, m, torch.bfloat16, 7)
    X = torch.randn(n, d_in, generator=gen, device=dev).bfloat16()
    ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(n, d_in, d_out), dev)

    def chain():
        Z = torch.empty(n, d_out, dtype=torch.bfloat16, device=dev)
        Y = libgq.gq_linear(X, codes, table, m, activation=act, Z=Z)
        y1 = libgq.gq_linear(X[:3], codes, table, m, activation=act)
        return [Y, Z, y1] + list(libgq.gq_linear_grad(Y, X, codes, table, m, ws, Z=Z, activation=act))
    want = chain()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = chain()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = chain()
    X2 = X.clone()
    X.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.count_nonzero(kept[0]) == 0
    X.copy_(X2)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, kept))
    libgq.gq_check()


def test_no_tokens(dev):
    gen, Q, codebook, codes, table, W = layer(dev, 64, 32, 4, torch.bfloat16, 2)
    X = torch.empty(0, 64, dtype=torch.bfloat16, device=dev)
    dY = torch.empty(0, 32, dtype=torch.bfloat16, device=dev)
    assert libgq.gq_linear(X, codes, table, 4).shape == (0, 32)
    ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(0, 64, 32), dev)
    _, dX, d_table, d_bias = libgq.gq_linear_grad(dY, X, codes, table, 4, ws)
    assert dX.shape == (0, 64) and torch.count_nonzero(d_table) == 0 and torch.count_nonzero(d_bias) == 0


def test_only_what_is_asked_for(dev):
    gen, Q, codebook, codes, table, W = layer(dev, 64, 32, 4, torch.bfloat16, 2)
    X = torch.randn(5, 64, device=dev).bfloat16()
    dY = torch.randn(5, 32, device=dev).bfloat16()
    launches = libgq.gq_launch_count()
    got = libgq.gq_linear_grad(dY, X, codes, table, 4, need_table=False, need_bias=False)
    assert got[0] is dY and got[2] is None and got[3] is None and libgq.gq_launch_count() - launches == 1
    ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(5, 64, 32), dev)
    full = libgq.gq_linear_grad(dY, X, codes, table, 4, ws)
    only = libgq.gq_linear_grad(dY, X, codes, table, 4, ws, need_x=False, need_table=False)
    assert only[1] is None and only[2] is None and torch.equal(only[3], full[3]) and torch.equal(got[1], full[1])


def test_binding_refuses(dev):
    gen, Q, codebook, codes, table, W = layer(dev, 64, 32, 4, torch.bfloat16, 2)
    X = torch.randn(5, 64, device=dev).bfloat16()
    with pytest.raises(ValueError, match="table"):
        libgq.gq_linear(X.half(), codes, table, 4)
    with pytest.raises(ValueError, match="codes"):
        libgq.gq_linear(X, codes[:, :16].contiguous(), table, 4)
    with pytest.raises(ValueError, match="residual"):
        libgq.gq_linear(X, codes, table, 4, residual=torch.zeros(5, 40, device=dev, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="bias"):
        libgq.gq_linear(X, codes, table, 4, bias=torch.zeros(32, device=dev))
    with pytest.raises(libgq.GQError, match="INVALID_ARG"):
        libgq.gq_linear(X, codes, table, 4, activation=7)
    with pytest.raises(libgq.GQError, match="ALIGNMENT"):
        libgq.gq_linear(torch.zeros(5, 68, device=dev, dtype=torch.bfloat16)[:, :64], codes, table, 4)
    with pytest.raises(libgq.GQError, match="WORKSPACE"):
        libgq.gq_linear_grad(torch.zeros(5, 32, device=dev, dtype=torch.bfloat16), X, codes, table, 4)
    with pytest.raises(ValueError, match="dZ"):
        libgq.gq_linear_grad(torch.zeros(5, 32, device=dev, dtype=torch.bfloat16), X, codes, table, 4, dZ=torch.zeros(5, 32, device=dev).bfloat16())


@pytest.mark.parametrize("n", [3, 20])
def test_rows_further_apart_than_32_bits(dev, n):
    """Activations, residual and outputs 2^28 elements apart: the last of 20 rows starts 10 GB behind the first."""
    ld, d_in, d_out, m = 1 << 28, 72, 64, 16
    gen, Q, codebook, codes, table, W = layer(dev, d_in, d_out, m, torch.bfloat16, 6)
    X = torch.randn(n, d_in, generator=gen, device=dev).bfloat16()
    R = torch.randn(n, d_out, generator=gen, device=dev).bfloat16()

    def far(t):
        f = torch.empty((n - 1) * ld + t.shape[1], dtype=t.dtype, device=dev).as_strided(t.shape, (ld, 1))
        return f.copy_(t)
    Y, Z = far(R), far(R)
    want_z = torch.empty_like(R)
    want = libgq.gq_linear(X, codes, table, m, residual=R, Z=want_z, activation=libgq.GQ_ACT_SILU)
    libgq.gq_linear(far(X), codes, table, m, residual=far(R), Y=Y, Z=Z, activation=libgq.GQ_ACT_SILU)
    assert torch.equal(Y, want) and torch.equal(Z, want_z)
    ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(n, d_in, d_out), dev)
    a = libgq.gq_linear_grad(R, X, codes, table, m, ws, Z=want_z, activation=libgq.GQ_ACT_SILU)
    b = libgq.gq_linear_grad(far(R), far(X), codes, table, m, ws, Z=Z, activation=libgq.GQ_ACT_SILU, dZ=far(R), dX=far(X))
    libgq.gq_check()
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("n,d_in,d_out,m", [(17, 2048, 248, 16), (40, 4096, 512, 16), (33, 16384, 256, 8), (100, 1032, 3000, 16), (256, 8192, 264, 4),
                                            (300, 2056, 520, 16), (150, 15320, 712, 4), (256, 512, 9472, 16)])
def test_few_tiles_share_the_contraction(dev, n, d_in, d_out, m):
    """Clusters of two, four and eight pairs, forward and backward (whose contraction is the other dimension)."""
    check_forward(dev, n, d_in, d_out, m, torch.float16, libgq.GQ_ACT_GELU, True, True, 8)
    check_backward(dev, n, d_out, d_in, m, torch.bfloat16, libgq.GQ_ACT_RELU, 8)


def test_two_calls_at_once(dev):
    """Calls on several streams, each with its own outputs and workspace, give what they give alone."""
    m, act = 16, libgq.GQ_ACT_GELU
    jobs = []
    for i, (n, d_in, d_out) in enumerate([(2, 4096, 1024), (40, 2048, 512), (900, 1032, 1408)]):
        gen, Q, codebook, codes, table, W = layer(dev, d_in, d_out, m, torch.bfloat16, i)
        X = torch.randn(n, d_in, generator=gen, device=dev).bfloat16()
        Z = torch.randn(n, d_out, generator=gen, device=dev).bfloat16()
        ws = libgq.alloc_workspace(libgq.gq_linear_grad_workspace_bytes(n, d_in, d_out), dev)
        jobs.append(lambda st=None, X=X, Z=Z, codes=codes, table=table, ws=ws: [libgq.gq_linear(X, codes, table, m, activation=act, stream=st)] + list(
            libgq.gq_linear_grad(Z, X, codes, table, m, ws, Z=Z, activation=act, stream=st)))
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = []
    for _ in range(4):
        got += [(i, job(s)) for i, (job, s) in enumerate(zip(jobs, streams))]
    torch.cuda.synchronize()
    libgq.gq_check()
    for i, outs in got:
        assert all(torch.equal(a, b) for a, b in zip(outs, want[i]))
