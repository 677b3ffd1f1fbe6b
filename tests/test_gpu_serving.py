"""attend_prefix, attend_mass and evict against a plain implementation in 64 bits.

Tolerances, per output element.  u = 2^-24 is half a step of fp32, n the tokens a query runs over, p their softmax weights:
  logit    |error| <= dl = (d + 8) u max_j sum_c |k_jc q_c| / sqrt d, plus 4 u of its own size and of the reference's (rounded products, the scale)
  weight   relative 2 dl (its own logit and the denominator's) + (n + 64) u (the sums) + 2^-16 (exp2; bf16: the two-number weights);
           + 2^-8 in the output of bf16 caches with more than 64 queries, whose weights are rounded to one bf16 number (half a step)
  out      that, times sum_j p_j |v_j|; and the rounding of the result: bf16 2^-8, fp32 u, relative
  lse      dl + (n + 64) u + 4 u |lse|
  mass     sum over the queries of p times the weights' bound, + 4 u of the result and (rows) u of the sum
A kept set is compared exactly.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def bk():
    import paper_2502_07861_amd as b
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return b


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _cache(gen, n_seq, stride, d, dtype, absent=0.1, poison=True):
    """Keys with outlier channels, values, weights of 1, 2 and 4; places without a token hold infinities and NaN."""
    K = torch.randn(n_seq, stride, d, generator=gen, device="cuda")
    K[:, :, :4] *= 6.0
    V = torch.randn(n_seq, stride, d, generator=gen, device="cuda")
    w = torch.exp2(torch.randint(0, 3, (n_seq, stride), generator=gen, device="cuda").float())
    gone = torch.rand(n_seq, stride, generator=gen, device="cuda") < absent
    if n_seq * stride:
        marks = torch.tensor([0.0, -1.0, float("nan"), -0.0], device="cuda")
        w = torch.where(gone, marks[torch.randint(0, 4, w.shape, generator=gen, device="cuda")], w)
        if poison:
            K[gone] = float("nan")
            V[gone] = float("inf")
    return K.to(dtype), V.to(dtype), w


def _attention(Q, K, V, w, sees=None):
    """One sequence in 64 bits: (out, lse, weights P, bound of a weight's relative error per query, dl)."""
    d = Q.shape[-1]
    live = w > 0
    K, V, Q = (torch.where(live[:, None], t.double(), 0.0) if t is not Q else t.double() for t in (K, V, Q))
    x = (Q @ K.T) / math.sqrt(d) + torch.where(live, w.double(), 1.0).log()
    see = live[None].expand_as(x)
    if sees is not None:
        see = see & (torch.arange(K.shape[0], device=Q.device)[None] < sees[:, None])
    x = x.masked_fill(~see, -math.inf)
    lse = torch.logsumexp(x, dim=1) if K.shape[0] else torch.full((Q.shape[0],), -math.inf, device=Q.device, dtype=torch.float64)
    finite = torch.where(torch.isinf(lse), 0.0, lse)
    P = torch.exp(x - finite[:, None])
    size = (Q.abs() @ K.abs().T / math.sqrt(d)).amax(dim=1) if K.shape[0] else torch.zeros_like(finite)
    big = torch.where(torch.isinf(x), 0.0, x.abs()).amax(dim=1) if K.shape[0] else torch.zeros_like(finite)
    dl = (d + 8) * U * size + 4 * U * (2 * big + 8)
    return P @ V, lse, P, 2 * dl + (K.shape[0] + 64) * U + 2.0 ** -16, dl, P @ V.abs()


def _check_out(out, lse, ref, dtype, n, what, rows=1):
    z, l, P, rel, dl, zabs = ref
    rel = rel + (2.0 ** -8 if dtype == BF16 and rows > 64 else 0.0)
    out, z = out.double().reshape(z.shape), z
    half = 2.0 ** -8 if dtype == BF16 else U
    tol = rel[:, None] * zabs + half * z.abs() * (1 + rel[:, None]) + 1e-30
    off = (out - z).abs()
    assert bool((off <= tol).all()), "%s: out off by %.3g of the bound" % (what, float((off / tol).max()))
    if lse is not None:
        got = lse.double().reshape(l.shape)
        none = torch.isinf(l)
        assert torch.equal(torch.isinf(got) & (got < 0), none), what
        off, tol = (got - l)[~none].abs(), (dl + (n + 64) * U + 4 * U * l.abs())[~none]
        assert bool((off <= tol).all()), "%s: lse off by %.3g of the bound" % (what, float((off / tol).max()))


PREFIX = [  # dtype, d, n_pre, fan, g, nq, count_p, count_s
    (BF16, 128, 1, 1, 1, 1, 1, 1), (BF16, 128, 2, 3, 4, 1, 63, 1), (BF16, 128, 3, 5, 2, 1, 64, 17), (BF16, 64, 2, 9, 4, 1, 65, 40),
    (BF16, 128, 2, 17, 4, 1, 257, 33), (BF16, 128, 1, 40, 4, 1, 1000, 64), (BF16, 64, 5, 33, 1, 1, 130, 0), (BF16, 128, 2, 2, 4, 1, 0, 70),
    (BF16, 128, 1, 13, 8, 5, 777, 5), (BF16, 64, 3, 1, 1, 130, 300, 31), (BF16, 128, 2, 300, 1, 1, 96, 3), (BF16, 128, 1, 2, 1, 1, 20001, 100),
    (F32, 128, 2, 3, 4, 1, 63, 1), (F32, 64, 3, 5, 2, 3, 1000, 33), (F32, 128, 1, 40, 4, 1, 200, 64), (F32, 64, 1, 7, 5, 1, 64, 0),
    (F32, 64, 2, 2, 1, 1, 0, 5), (F32, 128, 1, 1, 1, 1, 1, 0), (F32, 64, 2, 70, 2, 1, 129, 65), (BF16, 128, 600, 2, 1, 1, 130, 9), (BF16, 64, 100, 6, 4, 1, 70, 300),
    (F32, 128, 41, 13, 1, 1, 122, 31), (F32, 64, 3, 200, 2, 3, 200, 17), (BF16, 128, 4, 130, 4, 4, 64, 1), (BF16, 128, 520, 1, 3, 1, 33, 2000),
]


@pytest.mark.parametrize("dtype,d,n_pre,fan,g,nq,cp,cs", PREFIX)
def test_prefix(bk, dtype, d, n_pre, fan, g, nq, cp, cs):
    gen, n_seq = _gen(cp + 7 * cs + fan), n_pre * fan
    pre, own = _cache(gen, n_pre, cp + 3, d, dtype), _cache(gen, n_seq, cs + 2, d, dtype)
    Q = (2.0 * torch.randn(n_seq, g, nq, d, generator=gen, device="cuda")).to(dtype)
    p = bk.make_params(d, 64, 1, dtype, log_c=0.0)
    out, lse = bk.attend_prefix(p, pre, own, Q, count_prefix=cp, count_own=cs)
    for s in range(0, n_seq, max(1, n_seq // 40)):
        k = s % n_pre
        K, V, w = (torch.cat([a[k, :cp], b[s, :cs]]) for a, b in zip(pre, own))
        _check_out(out[s], lse[s], _attention(Q[s].reshape(-1, d), K, V, w), dtype, cp + cs, "sequence %d" % s, fan * g * nq)
    again, lse2 = bk.attend_prefix(p, pre, own, Q, count_prefix=cp, count_own=cs)
    assert torch.equal(out.view(torch.int16 if dtype == BF16 else torch.int32), again.view(torch.int16 if dtype == BF16 else torch.int32))
    assert torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fan", [6, 130])
def test_prefix_sequences_without_tokens(bk, dtype, fan):
    """Prefixes without a token, sequences without one, both, and neither."""
    gen, d, n_pre, cp, cs = _gen(3), 128, 4, 150, 70
    pre, own = _cache(gen, n_pre, cp, d, dtype), _cache(gen, n_pre * fan, cs, d, dtype)
    for k in (1, 2):
        pre[2][k], pre[0][k], pre[1][k] = 0.0, float("nan"), float("nan")
    for s in (0, 2, 5, 9, 23):
        own[2][s], own[0][s], own[1][s] = -1.0, float("inf"), float("-inf")
    Q = torch.randn(n_pre * fan, 4, 2, d, generator=gen, device="cuda").to(dtype)
    p = bk.make_params(d, 64, 1, dtype, log_c=0.0)
    out, lse = bk.attend_prefix(p, pre, own, Q)
    for s in range(24):
        K, V, w = (torch.cat([a[s % n_pre], b[s]]) for a, b in zip(pre, own))
        _check_out(out[s], lse[s], _attention(Q[s].reshape(-1, d), K, V, w), dtype, cp + cs, "sequence %d" % s, fan * 8)
    for s in (2, 5, 9):
        assert bool((out[s] == 0).all()) and bool((lse[s] == -math.inf).all())
    zeros, none = bk.attend_prefix(p, pre, own, Q, count_prefix=0, count_own=0)
    assert bool((zeros == 0).all()) and bool((none == -math.inf).all())
    assert bk.attend_prefix(p, pre, own, Q, lse=False)[1] is None


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fan", [1, 5, 12, 40, 200])
def test_an_infinite_value_shows_in_its_column(bk, dtype, fan):
    """... of every query that meets it, whatever shares its workgroup, and in no other."""
    gen, n_pre, cp, cs, d = _gen(fan), 2, 300, 40, 128
    pre, own = _cache(gen, n_pre, cp, d, dtype, absent=0.0), _cache(gen, n_pre * fan, cs, d, dtype, absent=0.0)
    for t in (pre[0], own[0]):
        t.mul_(0.05)                                    # (logits near 0: no weight vanishes)
    Q = (0.1 * torch.randn(n_pre * fan, 4, 1, d, generator=gen, device="cuda")).to(dtype)
    p = bk.make_params(d, 64, 1, dtype, log_c=0.0)
    ref, lse = bk.attend_prefix(p, pre, own, Q)
    pre[1][0, 170, 5] = float("inf")
    own[1][n_pre * fan - 1, 33, 77] = -float("inf")
    out, lse2 = bk.attend_prefix(p, pre, own, Q)
    assert torch.equal(lse, lse2) and bool((out[::2, :, :, 5] == float("inf")).all()) and bool((out[-1, :, :, 77] == -float("inf")).all())
    out[::2, :, :, 5], out[-1, :, :, 77] = ref[::2, :, :, 5], ref[-1, :, :, 77]
    assert torch.equal(out, ref)


MASS = [  # dtype, d, n_seq, count, g, nq, visible, decay
    (BF16, 128, 1, 1, 1, 1, None, 1.0), (BF16, 128, 3, 31, 4, 1, None, 0.5), (BF16, 128, 2, 33, 8, 1, None, 0.0), (BF16, 64, 2, 129, 4, 2, None, 1.0),
    (BF16, 128, 2, 1000, 4, 1, None, 0.9), (BF16, 128, 1, 9000, 16, 1, None, 1.0), (BF16, 128, 2, 700, 2, 37, 664, 0.0), (BF16, 128, 1, 260, 4, 260, 1, 0.5),
    (BF16, 64, 3, 200, 3, 200, 1, 1.0), (BF16, 128, 2, 127, 5, 70, -9, 1.0), (BF16, 128, 2, 64, 1, 40, -40, 1.0), (BF16, 128, 2, 64, 1, 40, -39, 1.0),
    (BF16, 128, 1, 128, 1, 5000, None, 0.25), (BF16, 64, 70, 300, 1, 1, None, 1.0), (BF16, 128, 1, 3000, 1, 300, 2701, 1.0),
    (F32, 64, 1, 1, 1, 1, None, 1.0), (F32, 128, 2, 130, 4, 1, None, 0.5), (F32, 64, 2, 333, 2, 37, -4, 0.5), (F32, 128, 1, 200, 2, 200, 1, 0.0),
    (F32, 64, 3, 4097, 4, 1, None, 1.0), (F32, 128, 2, 500, 1, 130, 371, 0.9), (F32, 64, 1, 70, 7, 70, 1, 1.0), (BF16, 128, 2, 500, 2, 10, -1000, 1.0),
    (BF16, 128, 2, 40, 2, 90, 1, 1.0), (BF16, 128, 9, 250, 3, 250, 1, 1.0), (BF16, 64, 50, 140, 2, 70, 71, 0.5), (F32, 128, 9, 150, 2, 100, 51, 1.0),
    (BF16, 128, 3, 2000, 1, 500, 1501, 1.0), (BF16, 64, 1, 640, 8, 640, -3, 0.0),
    (BF16, 128, 161, 2001, 4, 1, None, 0.5), (BF16, 64, 330, 77, 4, 2, None, 1.0), (F32, 128, 170, 777, 16, 1, None, 0.0), (F32, 64, 165, 1001, 1, 1, None, 1.0),
    (BF16, 128, 160, 8768, 4, 1, None, 1.0), (BF16, 128, 160, 9100, 4, 1, None, 1.0), (BF16, 128, 600, 1, 3, 1, None, 1.0), (BF16, 128, 5, 513, 2, 1, None, 1.0),
    (BF16, 128, 2, 64, 4, 40, -1000, 1.0), (F32, 64, 3, 300, 9, 30, -31, 0.5), (BF16, 128, 8, 420, 8, 420, 1, 1.0), (BF16, 64, 2, 530, 4, 300, 100, 1.0),
    (BF16, 128, 300, 400, 3, 1, None, 0.9), (BF16, 64, 520, 999, 4, 1, None, 1.0), (BF16, 64, 1500, 130, 1, 7, None, 0.0), (BF16, 128, 500, 4000, 4, 1, None, 1.0),
    (BF16, 128, 5, 512, 2, 8, None, 1.0), (F32, 128, 5, 256, 5, 3, None, 1.0), (F32, 128, 5, 257, 5, 3, None, 1.0), (BF16, 64, 5, 1024, 1, 7, None, 1.0),
]


def _check_mass(got, before, decay, refs, count, rows, what):
    P, rel = refs[2], refs[3]
    want = P.sum(dim=0)
    tol = (P * rel[:, None]).sum(dim=0) + rows * U * want
    if decay > 0:
        want = want + float(np.float32(decay)) * before[:count].double()
    tol = tol + 4 * U * want.abs() + 1e-30
    off = (got[:count].double() - want).abs()
    assert bool((off <= tol).all()), "%s: mass off by %.3g of the bound" % (what, float((off / tol).max()))


@pytest.mark.parametrize("dtype,d,n_seq,count,g,nq,visible,decay", MASS)
def test_mass(bk, dtype, d, n_seq, count, g, nq, visible, decay):
    gen = _gen(count + nq + n_seq)
    K, V, w = _cache(gen, n_seq, count + 5, d, dtype)
    Q = (2.0 * torch.randn(n_seq, g, nq, d, generator=gen, device="cuda")).to(dtype)
    before = torch.rand(n_seq, count + 5, generator=gen, device="cuda")
    p = bk.make_params(d, 64, 1, dtype, log_c=0.0)
    mass = before.clone() if decay > 0 else torch.full_like(before, float("nan"))        # (not read)
    into = torch.full_like(before, -7.0)
    out, lse, got = bk.attend_mass(p, K, V, w, Q, mass, count=count, visible=visible, decay=decay, mass_out=into)
    assert got is into and bool((into[:, count:] == -7.0).all())
    sees = None if visible is None else (visible + torch.arange(nq, device="cuda")).repeat(g)
    for s in range(0, n_seq, max(1, n_seq // 20)):
        ref = _attention(Q[s].reshape(-1, d), K[s, :count], V[s, :count], w[s, :count], sees)
        _check_out(out[s], lse[s], ref, dtype, count, "sequence %d" % s, g * nq)
        _check_mass(into[s], before[s], decay, ref, count, g * nq, "sequence %d" % s)
    # in place, and the same bits
    out2, _, got = bk.attend_mass(p, K, V, w, Q, mass, count=count, visible=visible, decay=decay, mass_out=mass, lse=False)
    assert got is mass and torch.equal(mass[:, :count], into[:, :count]) and torch.equal(out2, out)
    if decay > 0:
        assert torch.equal(mass[:, count:], before[:, count:])
    # without a mass to start from
    fresh = bk.attend_mass(p, K, V, w, Q, count=count, visible=visible)[2]
    zero = bk.attend_mass(p, K, V, w, Q, before, count=count, visible=visible, decay=0.0)[2]
    assert torch.equal(fresh, zero) and bool((fresh[:, count:] == 0).all())


@pytest.mark.parametrize("g,nq", [(2, 3), (4, 40)])
def test_places_that_no_query_sees_do_not_matter(bk, g, nq):
    gen = _gen(12)
    K, V, w = _cache(gen, 2, 300, 128, BF16)
    Q = torch.randn(2, g, nq, 128, generator=gen, device="cuda").to(BF16)
    p = bk.make_params(128, 64, 1, BF16, log_c=0.0)
    seen = 100 + nq - 1
    ref = bk.attend_mass(p, K, V, w, Q, visible=100)
    K[:, seen:], V[:, seen:] = float("nan"), float("inf")
    got = bk.attend_mass(p, K, V, w, Q, visible=100)
    assert all(torch.equal(a, b) for a, b in zip(got, ref)) and bool((got[2][:, seen:] == 0).all())


def test_mass_adds_up_to_the_queries(bk):
    """Every query that sees a token hands out a weight of 1."""
    gen = _gen(5)
    K, V, w = _cache(gen, 2, 600, 128, BF16)
    w[:, 0] = 1.0
    K[:, 0], V[:, 0] = 0.0, 0.0
    Q = torch.randn(2, 4, 600, 128, generator=gen, device="cuda").to(BF16)
    mass = bk.attend_mass(bk.make_params(128, 64, 1, BF16, log_c=0.0), K, V, w, Q, visible=-99)[2]
    # 500 positions of 4 heads each; a weight is off by its logit's and the sums' rounding: (136 + 600) u of sums near 100 at most
    torch.testing.assert_close(mass.double().sum(dim=1), torch.full((2,), 2000.0, device="cuda", dtype=torch.float64), rtol=2e-4, atol=0)


def test_mass_of_weights_far_apart(bk):
    """Weights of 2^-60 and 2^60 beside each other."""
    gen = _gen(6)
    K, V, w = _cache(gen, 1, 300, 128, F32, absent=0.0)
    w = torch.exp2(torch.randint(-60, 61, w.shape, generator=gen, device="cuda").float())
    Q = torch.randn(1, 2, 9, 128, generator=gen, device="cuda")
    out, lse, mass = bk.attend_mass(bk.make_params(128, 64, 1, F32, log_c=0.0), K, V, w, Q)
    ref = _attention(Q[0].reshape(-1, 128), K[0], V[0], w[0])
    _check_out(out[0], lse[0], ref, F32, 300, "far apart")
    _check_mass(mass[0], mass[0], 0.0, ref, 300, 18, "far apart")


def _kept(w, mass, count, keep, sink, recent):
    """Places that stay, ascending, by a sort over (class, -mass, place)."""
    w, m = w[:count].cpu().numpy(), mass[:count].cpu().numpy().astype(np.float64)
    m = np.where(np.isnan(m), -np.inf, m)
    place = np.arange(count)
    group = np.where(w > 0, np.where((place < sink) | (place >= count - recent), 0, 1), 2)
    order = np.lexsort((place, np.where(group == 1, -m, 0.0), group))[:keep]
    return np.sort(order[group[order] < 2])


def _check_evict(res, K, V, w, mass, idx, count, keep, sink, recent):
    for s in range(K.shape[0]):
        kept = _kept(w[s], mass[s], count, keep, sink, recent)
        n = len(kept)
        at = torch.from_numpy(kept).cuda()
        assert int(res["count"][s]) == n
        assert torch.equal(res["idx"][s, :n], idx[s][at] if idx is not None else at.int()), s
        for name, t in (("K", K), ("V", V), ("w", w), ("mass", mass)):
            bits = {2: torch.int16, 4: torch.int32}[t.element_size()]
            assert torch.equal(res[name][s, :n].view(bits), t[s][at].view(bits)), (s, name)
            assert bool((res[name][s, n:] == 0).all()), (s, name)
        assert bool((res["idx"][s, n:] == -1).all())


EVICT = [  # dtype, d, n_seq, count, extra stride, keep, sink, recent
    (BF16, 128, 1, 1, 0, 1, 0, 0), (BF16, 128, 3, 100, 7, 40, 4, 8), (BF16, 64, 2, 1025, 0, 512, 0, 100), (BF16, 128, 2, 5000, 3, 4999, 1, 1),
    (BF16, 128, 2, 5000, 3, 1, 0, 0), (BF16, 128, 2, 5000, 0, 1, 1, 0), (BF16, 64, 5, 4096, 0, 4096, 10, 10), (BF16, 128, 2, 20000, 0, 3000, 256, 256),
    (BF16, 64, 1, 70001, 0, 20000, 4, 100), (BF16, 64, 1, 300000, 5, 100001, 4, 100), (F32, 128, 2, 777, 1, 300, 0, 300), (F32, 64, 4, 1111, 9, 301, 3, 17), (F32, 64, 300, 65, 0, 31, 1, 1),
    (F32, 128, 1, 33000, 0, 8000, 8, 8), (BF16, 128, 2, 16384, 0, 384, 0, 5), (BF16, 128, 2, 16385, 1, 384, 4, 5), (BF16, 64, 3, 9000, 2, 768, 1, 1),
    (F32, 128, 2, 600, 0, 193, 1, 1),
]


@pytest.mark.parametrize("dtype,d,n_seq,count,extra,keep,sink,recent", EVICT)
@pytest.mark.parametrize("masses", ["spread", "ties", "odd", "equal"])
def test_evict(bk, dtype, d, n_seq, count, extra, keep, sink, recent, masses):
    gen, stride = _gen(count + keep), count + extra
    K, V, w = _cache(gen, n_seq, stride, d, dtype, absent=0.05)
    rand = lambda: torch.rand(n_seq, stride, generator=gen, device="cuda")
    mass = torch.exp(2.0 * torch.randn(n_seq, stride, generator=gen, device="cuda"))
    if masses == "ties":
        mass = torch.floor(rand() * 5.0)
    elif masses == "odd":
        odd = torch.tensor([0.0, -0.0, float("nan"), float("inf"), -float("inf"), -1.0, 1e-42, 3.0], device="cuda")
        mass = odd[torch.randint(0, 8, mass.shape, generator=gen, device="cuda")]
    elif masses == "equal":
        mass = torch.full_like(mass, 0.25)
        w = torch.where(rand() < 0.6, torch.zeros_like(w), w)              # often fewer tokens than are to be kept
    idx = torch.randint(0, 1 << 30, (n_seq, stride), generator=gen, device="cuda", dtype=torch.int32) if extra else None
    p = bk.make_params(d, 64, 1, dtype, log_c=0.0)
    ws = torch.randint(0, 255, (bk.evict_workspace_bytes(p, n_seq, count),), device="cuda", dtype=torch.uint8)
    res = bk.evict(p, K, V, w, mass, keep, n_sink=sink, n_recent=recent, count=count, idx=idx, workspace=ws)
    _check_evict(res, K, V, w, mass, idx, count, keep, sink, recent)


def test_evict_nothing(bk):
    p = bk.make_params(64, 64, 1, F32, log_c=0.0)
    K, w = torch.zeros(3, 40, 64, device="cuda"), torch.ones(3, 40, device="cuda")
    res = bk.evict(p, K, K, w, w, 0)
    assert bool((res["count"] == 0).all()) and res["K"].shape == (3, 0, 64)
    res = bk.evict(p, K, K, torch.zeros_like(w), w, 7, n_sink=2, n_recent=2)
    assert bool((res["count"] == 0).all()) and bool((res["idx"] == -1).all()) and bool((res["w"] == 0).all())


def test_offsets_past_32_bits(bk):
    """Sequences that start behind 4 GB, and one whose places do."""
    p = bk.make_params(64, 64, 1, BF16, log_c=0.0)
    gen, n_seq, stride, count = _gen(9), 5, 1 << 23, 90
    K = torch.empty(n_seq, stride, 64, device="cuda", dtype=BF16)          # 1 GiB a sequence
    V = torch.empty(n_seq, stride, 64, device="cuda", dtype=BF16)
    w = torch.zeros(n_seq, stride, device="cuda")
    k, v, x = _cache(gen, n_seq, count, 64, BF16)
    K[:, :count], V[:, :count], w[:, :count] = k, v, x
    Q = torch.randn(n_seq, 4, 1, 64, generator=gen, device="cuda").to(BF16)
    out, lse, mass = bk.attend_mass(p, K, V, w, Q, count=count)
    short = bk.attend_mass(p, k, v, x, Q)
    assert torch.equal(out, short[0]) and torch.equal(lse, short[1]) and torch.equal(mass[:, :count], short[2])
    both, lse2 = bk.attend_prefix(p, (K, V, w), (K, V, w), Q, count_prefix=count, count_own=0)
    _check_out(both[4], lse2[4], _attention(Q[4].reshape(-1, 64), k[4], v[4], x[4]), BF16, count, "behind 4 GB")
    res = bk.evict(p, K, V, w, mass, 33, count=count)
    _check_evict(res, k, v, x, mass[:, :count], None, count, 33, 0, 0)
    # one sequence of 5 GiB; its last places are the only tokens
    n = n_seq * stride
    K, V, w = K.view(1, n, 64), V.view(1, n, 64), w.view(1, n)
    w.zero_()
    K[0, n - count:], V[0, n - count:], w[0, n - count:] = k[0], v[0], x[0]
    Q = Q[:1]
    ref = _attention(Q[0].reshape(-1, 64), k[0], v[0], x[0])
    out, lse, mass = bk.attend_mass(p, K, V, w, Q)
    _check_out(out[0], lse[0], ref, BF16, n, "places behind 4 GB")
    assert bool((mass[0, :n - count] == 0).all())
    _check_mass(mass[0, n - count:], mass[0, :count], 0.0, ref, count, 4, "places behind 4 GB")
    res = bk.evict(p, K, V, w, mass, 40, n_recent=3)
    kept = _kept(w[0, n - count:], mass[0, n - count:], count, 40, 0, 3)
    assert res["idx"][0, :len(kept)].tolist() == [n - count + int(i) for i in kept]
    assert torch.equal(res["K"][0, :len(kept)], k[0][torch.from_numpy(kept).cuda()])


def _serve(bk, p, s):
    """A prompt judged by its last queries, brought down to its heaviest tokens, decoded on by several sessions."""
    _, _, mass = bk.attend_mass(p, s["K"], s["V"], s["w"], s["Qw"], visible=s["K"].shape[1] - s["Qw"].shape[2] + 1, workspace=s["ws"][0], mass_out=s["mass"])
    kept = bk.evict(p, s["K"], s["V"], s["w"], mass, 100, n_sink=4, n_recent=16, workspace=s["ws"][1])
    out, lse = bk.attend_prefix(p, (kept["K"], kept["V"], kept["w"]), s["own"], s["Q"], workspace=s["ws"][2])
    return mass, kept, out, lse


def _serve_state(bk, p, dtype, seed):
    gen, n_pre, fan, n, d = _gen(seed), 3, 7, 700, p.d
    K, V, w = _cache(gen, n_pre, n, d, dtype, absent=0.02)
    s = dict(K=K, V=V, w=w, Qw=torch.randn(n_pre, 4, 16, d, generator=gen, device="cuda").to(dtype), own=_cache(gen, n_pre * fan, 21, d, dtype),
             Q=torch.randn(n_pre * fan, 4, 1, d, generator=gen, device="cuda").to(dtype), mass=torch.empty(n_pre, n, device="cuda"))
    s["ws"] = [torch.empty(k, device="cuda", dtype=torch.uint8) for k in (bk.attend_mass_workspace_bytes(p, n_pre, n, 4, 16),
               bk.evict_workspace_bytes(p, n_pre, n), bk.attend_prefix_workspace_bytes(p, n_pre, n_pre * fan, 4, 1))]
    return s


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_together(bk, dtype):
    p = bk.make_params(128, 64, 1, dtype, log_c=0.0)
    s = _serve_state(bk, p, dtype, 1)
    mass, kept, out, lse = _serve(bk, p, s)
    sees = (700 - 16 + 1 + torch.arange(16, device="cuda")).repeat(4)
    for i in range(3):
        ref = _attention(s["Qw"][i].reshape(-1, 128), s["K"][i], s["V"][i], s["w"][i], sees)
        _check_mass(mass[i], mass[i], 0.0, ref, 700, 64, "prompt %d" % i)
    _check_evict(kept, s["K"], s["V"], s["w"], mass, None, 700, 100, 4, 16)
    for q in range(21):
        K, V, w = (torch.cat([kept[k][q % 3], t[q]]) for k, t in zip(("K", "V", "w"), s["own"]))
        _check_out(out[q], lse[q], _attention(s["Q"][q].reshape(-1, 128), K, V, w), dtype, 121, "session %d" % q)


def test_captured_and_on_another_stream(bk):
    """Two graphs that share workspaces, replayed in turn with eager work in between, new inputs included; and a side stream."""
    p = bk.make_params(128, 64, 1, BF16, log_c=0.0)
    states = [_serve_state(bk, p, BF16, 20 + i) for i in range(2)]
    states[1]["ws"] = states[0]["ws"]
    side = torch.cuda.Stream()
    want = [[t.clone() for t in (m, k["idx"], k["K"], o, l)] for m, k, o, l in (_serve(bk, p, s) for s in states)]
    same = lambda got, ref: all(torch.equal(a, b) for a, b in zip(got, ref))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m, k, o, l = _serve(bk, p, states[0])
    side.synchronize()
    assert same((m, k["idx"], k["K"], o, l), want[0])
    graphs, held = [], []
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m, k, o, l = _serve(bk, p, s)
        graphs.append(g)
        held.append((m, k["idx"], k["K"], o, l))
    for turn in range(4):
        for i, g in enumerate(graphs):
            for t in held[i]:
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert same(held[i], want[i]), (turn, i)
            m, k, o, l = _serve(bk, p, states[1 - i])                       # eager work on the same workspaces
            assert same((m, k["idx"], k["K"], o, l), want[1 - i])
    # new queries in the captured buffers
    other = _serve_state(bk, p, BF16, 77)
    for name in ("K", "V", "w", "Qw", "Q"):
        states[0][name].copy_(other[name])
    m, k, o, l = _serve(bk, p, states[0])
    fresh = [t.clone() for t in (m, k["idx"], k["K"], o, l)]
    graphs[0].replay()
    torch.cuda.synchronize()
    assert same(held[0], fresh)


def test_whole_sequences_captured(bk):
    """Logits of whole sequences in more LDS than a launch has by default, eviction in one launch, sequences of few own tokens: from a graph."""
    p = bk.make_params(128, 64, 1, BF16, log_c=0.0)
    gen, n, count = _gen(50), 256, 5000
    K, V, w = _cache(gen, n, count, 128, BF16)
    Q = torch.randn(n, 4, 1, 128, generator=gen, device="cuda").to(BF16)
    ws = [torch.empty(k, device="cuda", dtype=torch.uint8) for k in (bk.attend_mass_workspace_bytes(p, n, count, 4, 1), bk.evict_workspace_bytes(p, n, count),
                                                                     bk.attend_prefix_workspace_bytes(p, 8, 1024, 4, 1))]
    own, Qo = _cache(gen, 1024, 9, 128, BF16), torch.randn(1024, 4, 1, 128, generator=gen, device="cuda").to(BF16)

    def step(mass):
        out, lse, got = bk.attend_mass(p, K, V, w, Q, mass, decay=0.5, workspace=ws[0])
        kept = bk.evict(p, K, V, w, got, 300, n_sink=4, n_recent=64, workspace=ws[1])
        pre = tuple(kept[k][:8] for k in ("K", "V", "w"))
        z, l2 = bk.attend_prefix(p, pre, own, Qo, workspace=ws[2])
        return out, lse, got, kept["idx"], kept["V"], z, l2

    mass = torch.rand(n, count, generator=gen, device="cuda")
    want = [t.clone() for t in step(mass)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(mass)
    for turn in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), turn
        assert all(torch.equal(a, b) for a, b in zip(step(mass), want)), turn


def test_caches_of_the_streaming_handle(bk):
    """A Cache's views are taken as they are: prefix decode and masses over the handle's own storage, against attend."""
    p = bk.make_params(128, 64, 1, BF16, log_c=-5.0, seed=4)
    gen, n_seq = _gen(31), 4
    cache = bk.Cache(p, n_seq, max_tokens=600)
    K, V, _ = _cache(gen, n_seq, 512, 128, BF16, absent=0.0)
    cache.prefill(p, K, V)
    for i in range(5):
        cache.append_token(K[:, i].contiguous(), V[:, i].contiguous())
    Q = torch.randn(n_seq, 4, 1, 128, generator=gen, device="cuda").to(BF16)
    ref, lse = cache.attend(Q)
    Kc, Vc, wc = cache.views()
    out, lse2, mass = bk.attend_mass(p, Kc, Vc, wc, Q, count=cache.count)
    # both round the same sums differently: half a step of bf16 each, and the bounds of two passes over 261 tokens on the logarithm
    torch.testing.assert_close(out.double(), ref.double(), rtol=2 * 2.0 ** -8, atol=2.0 ** -12)
    torch.testing.assert_close(lse2, lse, rtol=0, atol=1e-4)
    out, lse2 = bk.attend_prefix(p, (Kc, Vc, wc), (Kc, Vc, wc), Q, count_prefix=cache.count, count_own=0)
    torch.testing.assert_close(out.double(), ref.double(), rtol=2 * 2.0 ** -8, atol=2.0 ** -12)
    kept = bk.evict(p, Kc, Vc, wc, mass, 100, n_recent=5, count=cache.count)
    cache.load(kept["K"], kept["V"], kept["w"])
    assert cache.count == 100
    cache.close()


def test_ablation_compares_eviction(bk):
    """The study's eviction columns: the kept sets by the formulas, the estimate over them, and the error formula on top."""
    from paper_2502_07861_amd import ablation
    res = ablation.run_evict(seeds=1, n_mid=1024, n_seq=2, nq=8, rounds=(1, 2), keep_outputs=True)
    n, q = res["K"].shape[1], res["judge"].reshape(2, -1, 128)
    ones = torch.ones(n, device="cuda")
    for row in res["rows"]:
        last = row["last"]
        for s in range(2):
            ref = _attention(q[s], res["K"][s], res["V"][s], ones)
            _check_mass(last["mass"][s], last["mass"][s], 0.0, ref, n, 16, "sequence %d" % s)
            kept = _kept(ones, last["mass"][s], n, row["kept"], ablation.N_SINK, ablation.N_RECENT)
            assert last["idx"][s].tolist() == kept.tolist()
            at = torch.from_numpy(kept).cuda()
            _check_out(last["z"][s], None, _attention(res["ask"][s].reshape(-1, 128), res["K"][s][at], res["V"][s][at], ones[at]), BF16, len(kept), "rate " + row["rate"])
        assert row["kept"] == 512 + (1024 >> (1 if row["rate"] == "1/2" else 2)) and row["evict"] == ablation.relative_error(last["z"], res["exact"])
    assert len(ablation.evict_table(res).splitlines()) == 4


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("g,cs", [(1, 1), (4, 31), (3, 32), (32, 33), (5, 64), (8, 127), (2, 255)])
def test_prefix_many_sequences_of_few_tokens(bk, dtype, d, g, cs):
    """More sequences than compute units, a few own tokens each, some of them absent, some sequences without one."""
    gen, n_pre, fan, cp = _gen(g + cs), 3, 101 if cs < 128 else 342, 70
    pre, own = _cache(gen, n_pre, cp, d, dtype), _cache(gen, n_pre * fan, cs + 1, d, dtype)
    own[2][5:9], own[0][5:9], own[1][5:9] = 0.0, float("nan"), float("nan")
    Q = torch.randn(n_pre * fan, g, 1, d, generator=gen, device="cuda").to(dtype)
    p = bk.make_params(d, 64, 1, dtype, log_c=0.0)
    out, lse = bk.attend_prefix(p, pre, own, Q, count_own=cs)
    alone, lse2 = bk.attend_prefix(p, pre, own, Q, count_prefix=0, count_own=cs)
    for s in list(range(12)) + [100, 301, 302]:
        K, V, w = (torch.cat([a[s % n_pre], b[s, :cs]]) for a, b in zip(pre, own))
        _check_out(out[s], lse[s], _attention(Q[s].reshape(-1, d), K, V, w), dtype, cp + cs, "sequence %d" % s, fan * g)
        _check_out(alone[s], lse2[s], _attention(Q[s].reshape(-1, d), own[0][s, :cs], own[1][s, :cs], own[2][s, :cs]), dtype, cs, "sequence %d alone" % s)
