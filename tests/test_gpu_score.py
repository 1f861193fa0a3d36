"""Token log probabilities, entropies, alternatives and their gradient against 64 bits.

Tolerances, derived: u = 2^-24.  A term exp(x - m) is off by at most (2 |x - m| + 4) u relative (the subtraction, the product with
log2 e, the exponential's two units in the last place); a thread adds up at most ceil(vocab / 512) + 8 terms one after the other and
the trees above it at most 17.  With D the largest |x - m| of a term that matters (a term below 2^-26 of the sum changes nothing at
this size; 20 is put in for it) L is off by at most (vocab / 512 + 25 + 2 * 20 + 4) u, plus its own rounding; the entropy by that
times (1 + 2 E|x - m|) with E|x - m| <= entropy + L; logp by L's error and the roundings of two subtractions."""
import pytest
import torch

from paper_2505_07004_b200 import api as libgq

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
INF = float("inf")
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    return torch.device("cuda:0")


def make(dev, n, vocab, dtype, seed, spread=3.0, pad=0, offset=0):
    """Logits as a view of a larger buffer: leading dimension vocab + pad, starting `offset` elements into it."""
    gen = torch.Generator(device=dev).manual_seed(seed)
    buf = torch.full((offset + n * (vocab + pad) + 16,), float("nan"), device=dev, dtype=dtype)
    x = buf[offset:offset + n * (vocab + pad)].view(n, vocab + pad)[:, :vocab]
    x.copy_(spread * torch.randn(n, vocab, generator=gen, device=dev))
    t = torch.randint(0, vocab, (n,), generator=gen, device=dev)
    return x, t, gen


def reference(x, t, top):
    x = x.double()
    vocab = x.shape[1]
    m = x.amax(1)
    none = m == -INF
    shifted = torch.where(none[:, None], -INF, x - m[:, None])           # exact where it matters, also next to the lowest value
    L = torch.where(none, 0.0, torch.logsumexp(shifted, 1))
    logp_all = shifted - L[:, None]
    p = logp_all.exp()
    entropy = -torch.special.xlogy(p, p).sum(1)
    counted = (t >= 0) & (t < vocab)
    logp = torch.where(counted, logp_all.gather(1, torch.where(counted, t, 0)[:, None])[:, 0], 0.0)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    return m, L, logp, entropy, logp_all.gather(1, order), order


def close(got, want, tol):
    got = got.double()
    same = (got == want) | (got.isnan() & want.isnan())
    assert bool((same | ((got - want).abs() <= tol)).all()), ((got - want).abs() / tol).nan_to_num().max().item()


def check_scores(x, t, top):
    logp, entropy, stats, top_logp, top_ids = libgq.gq_token_logprobs(x, t, top=top)
    m, L, logp_w, ent_w, tl_w, ti_w = reference(x, t, top)
    tol = (x.shape[1] / 512 + 69) * U
    assert torch.equal(stats[:, 0].double(), m)
    close(stats[:, 1], L, tol + 2 * U * L.abs())
    close(logp, logp_w, tol + 2 * U * (logp_w.abs() + L.abs()))
    close(entropy, ent_w, tol * (1 + 2 * (ent_w + L)) + 2 * U * ent_w)
    if top:
        assert torch.equal(top_ids.long(), ti_w)
        close(top_logp, tl_w, tol + 2 * U * (tl_w.abs() + L[:, None].abs()))
    else:
        assert top_logp is None and top_ids is None
    return logp, entropy, stats


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("n,vocab,top", [(1, 1, 1), (2, 2, 2), (3, 7, 7), (2, 8, 3), (5, 9, 0), (1, 511, 32), (3, 512, 1), (2, 4095, 20), (1, 32000, 5),
                                         (7, 32000, 20), (300, 1000, 4), (150, 50001, 32), (1, 160000, 32), (33, 8200, 2), (1200, 33, 32), (1300, 4099, 5),
                                         (1190, 9000, 32), (1184, 64, 0)])
def test_scores_match_64_bits(dev, dtype, n, vocab, top):
    x, t, _ = make(dev, n, vocab, DT[dtype], seed=n + vocab)
    check_scores(x, t, top)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 3), (5, 0), (8, 7), (24, 5)])
def test_strides_and_unaligned_rows(dev, dtype, pad, offset):
    x, t, gen = make(dev, 6, 2061, DT[dtype], seed=pad, pad=pad, offset=offset)
    logp, entropy, stats = check_scores(x, t, 9)
    check_gradient(x, t, stats, entropy, gen, pad_out=offset, offset_out=pad)


@pytest.mark.parametrize("dtype", sorted(DT))
def test_rows_of_equal_logits_give_the_first_indices(dev, dtype):
    x = torch.full((3, 9001), 1.25, device=dev, dtype=DT[dtype])
    x[1, 5000:] = 2.5
    x[2] = 0.0
    x[2, 1::2] = -0.0                                     # both zeros are one value
    check_scores(x, torch.tensor([0, 1, 9000], device=dev), 32)
    x = x.repeat(400, 1)                                  # rows for a CTA of the smaller size each
    check_scores(x, torch.arange(1200, device=dev) * 7, 32)


@pytest.mark.parametrize("dtype", sorted(DT))
def test_few_values_with_many_ties(dev, dtype):
    gen = torch.Generator(device=dev).manual_seed(4)
    x = torch.randint(0, 3, (40, 33333), generator=gen, device=dev).to(DT[dtype])
    check_scores(x, torch.randint(0, 33333, (40,), generator=gen, device=dev), 32)


@pytest.mark.parametrize("dtype", sorted(DT))
def test_masked_logits(dev, dtype):
    x, t, gen = make(dev, 8, 5003, DT[dtype], seed=9)
    low = torch.finfo(DT[dtype]).min
    x[0] = -INF                                           # nothing left
    x[1, 1:] = -INF                                       # one token left
    x[2, torch.rand(5003, generator=gen, device=dev) < 0.9] = -INF
    x[3] = low                                            # masks of the lowest value, everywhere and nearly everywhere
    x[4, 17:] = low
    x[5, ::2] = -INF
    x[6, :5000] = -INF
    x[7, 40:] = -INF
    t[2] = int((x[2] == -INF).nonzero()[0])               # a ruled-out target
    t[1], t[4], t[6] = 0, 3, 5002
    for top in (0, 1, 5, 32):
        check_scores(x.repeat(150, 1), t.repeat(150), top)              # rows for a CTA of the smaller size each
        logp, entropy, stats = check_scores(x, t, top)
    assert stats[0].tolist() == [-INF, 0.0] and entropy[0] == 0 and logp[0] == -INF
    assert logp[1] == 0 and logp[2] == -INF
    grad = check_gradient(x, t, stats, entropy, gen)
    assert torch.count_nonzero(grad[0]) == 0


def test_not_numbers(dev):
    x, t, _ = make(dev, 4, 3000, torch.float32, seed=3)
    x[0, 2999] = float("nan")
    x[1, 0] = INF
    x[2] = float("nan")
    x[2, 7] = 1.0
    logp, entropy, stats, top_logp, top_ids = libgq.gq_token_logprobs(x, t, top=4)
    assert logp[:3].isnan().all() and entropy[:3].isnan().all() and stats[:3, 1].isnan().all()
    assert torch.equal(top_ids[0].long(), torch.sort(x[0, :2999], descending=True, stable=True).indices[:4])
    assert top_ids[1, 0] == 0 and top_ids[2].tolist() == [7, -1, -1, -1]
    check = libgq.gq_token_logprobs(x[3:], t[3:], top=4)  # the row beside them is what it is alone
    assert torch.equal(logp[3:], check[0]) and torch.equal(top_ids[3:], check[4])


def check_gradient(x, t, stats, entropy, gen, with_logp=True, with_entropy=True, pad_out=0, offset_out=0):
    n, vocab = x.shape
    dev = x.device
    dl = torch.randn(n, generator=gen, device=dev) if with_logp else None
    de = torch.randn(n, generator=gen, device=dev) if with_entropy else None
    ld = vocab + pad_out
    buf = torch.full((offset_out + (n + 1) * ld,), 77.0, dtype=x.dtype, device=dev)
    out = buf[offset_out:].view(n + 1, ld)
    got = libgq.gq_token_logprobs_grad(x, t, stats, entropy, dl, de, d_logits=out[:n, :vocab])
    assert bool((out[n] == 77.0).all()) and bool((out[:, vocab:] == 77.0).all()) and bool((buf[:offset_out] == 77.0).all())
    xd, sd = x.double(), stats.double()
    none = sd[:, :1] == -INF
    logp = torch.where(none, -INF, (xd - sd[:, :1]) - sd[:, 1:])
    p = logp.exp()
    counted = (t >= 0) & (t < vocab)
    w = torch.where(counted, dl.double(), 0.0)[:, None] if with_logp else torch.zeros(n, 1, device=dev, dtype=torch.float64)
    h = de.double()[:, None] if with_entropy else torch.zeros_like(w)
    hit = torch.zeros_like(xd)
    hit.scatter_(1, torch.where(counted, t, 0)[:, None], 1.0)
    want = w * (hit * counted[:, None] - p) - h * (torch.special.xlogy(p, p) + p * entropy.double()[:, None])
    want = torch.where(none, 0.0, want)
    # two subtractions, a product and the exponential give p to (2 |x - m| + 2 L + 4) u; the sums of products a few u more; a p below
    # 2^-126 is taken as 0
    bend = torch.where(p > 0, (2 * (xd - sd[:, :1]).abs() + 2 * sd[:, 1:] + 8) * U, 0.0)
    size = p * (w.abs() + h.abs() * (logp.clamp_min(-200.0).abs() + entropy.double()[:, None].abs()))
    size = torch.where(none, 0.0, size)
    lost = torch.where(p < 2.0 ** -126, size, 0.0)
    tol = lost + 2 * bend * size + 4 * U * (size + w.abs() * hit) + want.abs() * (torch.finfo(x.dtype).eps / 2)
    tol = tol + (torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps if x.dtype != torch.float32 else 2.0 ** -126)
    tol = tol * 1.01
    assert bool(((got.double() - want).abs() <= tol).all()), ((got.double() - want).abs() / tol).max().item()
    return got


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("n,vocab", [(1, 1), (2, 7), (3, 8), (4, 4097), (3, 32000), (70, 1001), (5, 50001)])
@pytest.mark.parametrize("parts", ["logp", "entropy", "both"])
def test_gradient_matches_the_formula(dev, dtype, n, vocab, parts):
    x, t, gen = make(dev, n, vocab, DT[dtype], seed=vocab)
    t[0] = -100
    _, entropy, stats, _, _ = libgq.gq_token_logprobs(x, t)
    grad = check_gradient(x, t, stats, entropy, gen, with_logp=parts != "entropy", with_entropy=parts != "logp")
    if parts == "logp":
        assert torch.count_nonzero(grad[0]) == 0          # its token does not count


def test_gradient_matches_differences(dev):
    """Central differences of the library's own outputs: with step e the truncation is e^2 / 6 times a third derivative that is at most
    about 6 |w| p, and an output is off by 1e-5 at most at this size."""
    x, t, gen = make(dev, 2, 50, torch.float32, seed=5)
    w, h, e = torch.tensor([0.7, -1.3], device=dev), torch.tensor([0.4, 0.9], device=dev), 2.0 ** -6
    _, entropy, stats, _, _ = libgq.gq_token_logprobs(x, t)
    grad = libgq.gq_token_logprobs_grad(x, t, stats, entropy, w, h)

    def total(x):
        lp, en, _, _, _ = libgq.gq_token_logprobs(x, t)
        return (w * lp + h * en).double()
    for j in range(50):
        up, down = x.clone(), x.clone()
        up[:, j] += e
        down[:, j] -= e
        numeric = (total(up) - total(down)) / (up[:, j] - down[:, j]).double()
        assert bool(((numeric - grad[:, j].double()).abs() <= 1e-5 / e + 20 * e * e).all())


def test_rows_without_weight_are_not_read(dev):
    x, t, gen = make(dev, 3, 4000, torch.bfloat16, seed=8)
    _, entropy, stats, _, _ = libgq.gq_token_logprobs(x, t)
    x[1] = float("nan")
    t[1] = 4000                                           # outside the vocabulary
    grad = libgq.gq_token_logprobs_grad(x, t, stats, None, torch.ones(3, device=dev))
    assert torch.count_nonzero(grad[1]) == 0 and bool(grad.isfinite().all())


def test_streams_and_graphs(dev):
    x, t, _ = make(dev, 5, 32000, torch.bfloat16, seed=2)
    d = torch.randn(5, device=dev)

    def both():
        logp, entropy, stats, tl, ti = libgq.gq_token_logprobs(x, t, top=7)
        return [logp, entropy, stats, tl, ti, libgq.gq_token_logprobs_grad(x, t, stats, entropy, d, d)]
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = both()
    keep_x = x.clone()
    x.copy_(torch.randn(5, 32000, device=dev))
    graph.replay()
    again = both()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, again))
    x.copy_(keep_x)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, want))


def test_empty_batch(dev):
    logp, entropy, stats, tl, ti = libgq.gq_token_logprobs(torch.empty(0, 100, device=dev), torch.empty(0, dtype=torch.int64, device=dev), top=3)
    assert logp.shape == (0,) and entropy.shape == (0,) and stats.shape == (0, 2) and tl.shape == (0, 3) and ti.shape == (0, 3)


def test_binding_refuses(dev):
    x, t, _ = make(dev, 3, 100, torch.float32, seed=1)
    with pytest.raises(ValueError, match="targets"):
        libgq.gq_token_logprobs(x, t.int())
    with pytest.raises(ValueError, match="targets"):
        libgq.gq_token_logprobs(x, t[:2])
    with pytest.raises(ValueError, match="contiguous"):
        libgq.gq_token_logprobs(x.t())
    with pytest.raises(libgq.GQError, match="INVALID_ARG"):
        libgq.gq_token_logprobs(x[:, :5], top=6)
    with pytest.raises(libgq.GQError, match="UNSUPPORTED_SHAPE"):
        libgq.gq_token_logprobs(x, top=33)
    with pytest.raises(ValueError, match="stats"):
        libgq.gq_token_logprobs_grad(x, t, torch.zeros(3, device=dev), None, torch.zeros(3, device=dev))


def test_rows_further_apart_than_32_bits(dev):
    """Three rows of bf16 logits 2^30 elements apart: the last one starts 4 GB behind the first."""
    ld, vocab = 1 << 30, 3001
    buf = torch.empty(2 * ld + vocab, dtype=torch.bfloat16, device=dev)
    x = buf.as_strided((3, vocab), (ld, 1))
    x.copy_(3 * torch.randn(3, vocab, device=dev))
    t = torch.tensor([5, 3000, 17], device=dev)
    logp, entropy, stats = check_scores(x, t, 5)
    out = torch.empty_like(buf).as_strided((3, vocab), (ld, 1))
    d = torch.ones(3, device=dev)
    assert torch.equal(libgq.gq_token_logprobs_grad(x, t, stats, entropy, d, d, d_logits=out), libgq.gq_token_logprobs_grad(x.contiguous(), t, stats, entropy, d, d))


def test_two_calls_at_once(dev):
    xs = [make(dev, n, 40000, torch.float32, seed=n)[:2] for n in (3, 1500)]
    want = [libgq.gq_token_logprobs(x, t, top=9) for x, t in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[] for _ in xs]
    for _ in range(5):
        for i, (s, (x, t)) in enumerate(zip(streams, xs)):
            got[i].append(libgq.gq_token_logprobs(x, t, top=9, stream=s))
    torch.cuda.synchronize()
    for i in range(len(xs)):
        assert all(torch.equal(a, b) for run in got[i] for a, b in zip(run, want[i]))


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("n", [6, 1206])
def test_values_next_to_the_ends_of_the_type(dev, dtype, n):
    """Rows far from zero, up to the largest and down to the lowest finite values, with -inf beside them: only differences count."""
    big = torch.finfo(DT[dtype]).max
    x, t, gen = make(dev, n, 2000, DT[dtype], seed=n, spread=2.0)
    base = torch.tensor([0.0, 3.0e4, -6.4e4, 1.0e3, -1.0e3, 6.0e4] if dtype == "fp16" else [0.0, 1.0e20, -1.0e29, 3.0e4, -2.0e31, 1.0e36], device=dev)
    x += base.repeat(n // 6)[:, None].to(x.dtype)
    x[1, ::3] = -INF
    x[2, 1::2] = -INF
    x[3, :1999] = -big
    x[4, 5:] = -big
    x[5, 7] = big
    x[0, 100:] = -INF
    t[0], t[1], t[2], t[3], t[4], t[5] = 5, 1, 0, 1999, 3, 7
    _, entropy, stats = check_scores(x, t, 3)
    check_gradient(x, t, stats, entropy, gen)
