"""attend_prefix, attend_mass and evict where their arguments are unusual: against a plain implementation in 64 bits, with the bounds of
test_gpu_serving.py."""
import math

import pytest
import torch

from test_gpu_serving import BF16, F32, _attention, _cache, _check_evict, _check_mass, _check_out, _gen, bk  # noqa: F401  (bk: a fixture)

pytestmark = pytest.mark.gpu


def _paired(gen, n_seq, n, d, dtype):
    """Tokens in pairs: the same key, opposite values, weights 1 and 1 + delta, delta in 2^-9 .. 2^-7.  The answer is the small difference that
    deltas leave, so the rounding of the weights shows in it and its own rounding does not."""
    K = (0.2 * torch.randn(n_seq, n // 2, d, generator=gen, device="cuda")).to(dtype).repeat_interleave(2, dim=1)
    V = torch.randn(n_seq, n // 2, d, generator=gen, device="cuda").to(dtype).repeat_interleave(2, dim=1)
    V[:, 1::2] *= -1.0
    w = torch.ones(n_seq, n, device="cuda")
    w[:, 1::2] += torch.exp2(-9.0 + 2.0 * torch.rand(n_seq, n // 2, generator=gen, device="cuda"))
    return K, V, w


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("n_pre,fan,g,nq", [(2, 1, 1, 1), (2, 3, 4, 1), (2, 8, 4, 2), (2, 33, 4, 5), (100, 15, 4, 1), (100, 33, 4, 1), (40, 33, 4, 5)])
def test_an_answer_is_as_exact_in_any_company(bk, dtype, d, n_pre, fan, g, nq):  # noqa: F811
    """The weights' 2^-16 holds whatever the number of queries that share a prefix."""
    gen, cp, cs = _gen(fan + d), 200, 40
    pre, own = _paired(gen, n_pre, cp, d, dtype), _paired(gen, n_pre * fan, cs, d, dtype)
    Q = (0.2 * torch.randn(n_pre * fan, g, nq, d, generator=gen, device="cuda")).to(dtype)
    out, lse = bk.attend_prefix(bk.make_params(d, 64, 1, dtype, log_c=0.0), pre, own, Q)
    for s in range(0, n_pre * fan, max(1, n_pre * fan // 40)):
        K, V, w = (torch.cat([a[s % n_pre], b[s]]) for a, b in zip(pre, own))
        _check_out(out[s], lse[s], _attention(Q[s].reshape(-1, d), K, V, w), dtype, cp + cs, "sequence %d" % s)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("n_seq,g,nq,visible", [(2, 4, 1, None), (2, 4, 20, None), (3, 4, 64, 137), (200, 4, 32, None), (150, 4, 64, 137), (40, 4, 200, 1)])
def test_an_answer_is_as_exact_whatever_is_asked_beside_it(bk, dtype, d, n_seq, g, nq, visible):  # noqa: F811
    gen, count = _gen(nq + d), 200
    K, V, w = _paired(gen, n_seq, count, d, dtype)
    Q = (0.2 * torch.randn(n_seq, g, nq, d, generator=gen, device="cuda")).to(dtype)
    out, lse, mass = bk.attend_mass(bk.make_params(d, 64, 1, dtype, log_c=0.0), K, V, w, Q, visible=visible)
    sees = None if visible is None else (visible + torch.arange(nq, device="cuda")).repeat(g)
    for s in range(0, n_seq, max(1, n_seq // 10)):
        ref = _attention(Q[s].reshape(-1, d), K[s], V[s], w[s], sees)
        _check_out(out[s], lse[s], ref, dtype, count, "sequence %d" % s)
        _check_mass(mass[s], mass[s], 0.0, ref, count, g * nq, "sequence %d" % s)


# Token weights: subnormal ones are tokens like all others.  "far": beside weights up to 2^60; "small": subnormal ones alone; "equal": all the same
# subnormal number; "few": one subnormal token in a tile of ordinary ones.
def _odd_weights(gen, shape, kind):
    rand = lambda: torch.rand(*shape, generator=gen, device="cuda")
    if kind == "equal":
        return torch.full(shape, 2.0 ** -130, device="cuda")
    small = (1.0 + torch.floor(rand() * 1e6)) * 2.0 ** -149
    if kind == "small":
        return small
    if kind == "few":
        return torch.where(rand() < 0.02, small, torch.ones(shape, device="cuda"))
    far = torch.exp2(torch.floor(rand() * 121.0) - 60.0)
    return torch.where(rand() < 0.3, small, far)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("kind", ["far", "small", "equal", "few"])
@pytest.mark.parametrize("n_seq,count,g,nq,visible", [(2, 300, 4, 1, None), (2, 3000, 4, 1, None), (200, 100, 4, 1, None), (2, 300, 4, 9, None),
                                                      (1, 300, 4, 40, None), (2, 130, 1, 130, 1), (300, 40, 4, 7, None)])
def test_mass_of_subnormal_weights(bk, dtype, d, kind, n_seq, count, g, nq, visible):  # noqa: F811
    gen = _gen(count + nq)
    K, V, w = _cache(gen, n_seq, count, d, dtype, absent=0.0)
    w = _odd_weights(gen, (n_seq, count), kind)
    Q = torch.randn(n_seq, g, nq, d, generator=gen, device="cuda").to(dtype)
    out, lse, mass = bk.attend_mass(bk.make_params(d, 64, 1, dtype, log_c=0.0), K, V, w, Q, visible=visible)
    sees = None if visible is None else (visible + torch.arange(nq, device="cuda")).repeat(g)
    for s in range(0, n_seq, max(1, n_seq // 5)):
        ref = _attention(Q[s].reshape(-1, d), K[s], V[s], w[s], sees)
        _check_out(out[s], lse[s], ref, dtype, count, "sequence %d" % s)
        _check_mass(mass[s], mass[s], 0.0, ref, count, g * nq, "sequence %d" % s)


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("kind", ["far", "small", "equal", "few"])
@pytest.mark.parametrize("n_pre,fan,g", [(2, 3, 4), (1, 9, 4), (1, 40, 4), (150, 2, 1)])
def test_prefix_of_subnormal_weights(bk, dtype, d, kind, n_pre, fan, g):  # noqa: F811
    gen, n_seq, cp, cs = _gen(fan), n_pre * fan, 150, 50
    pre, own = list(_cache(gen, n_pre, cp, d, dtype, absent=0.0)), list(_cache(gen, n_seq, cs, d, dtype, absent=0.0))
    pre[2], own[2] = _odd_weights(gen, (n_pre, cp), kind), _odd_weights(gen, (n_seq, cs), kind)
    Q = torch.randn(n_seq, g, 1, d, generator=gen, device="cuda").to(dtype)
    p = bk.make_params(d, 64, 1, dtype, log_c=0.0)
    out, lse = bk.attend_prefix(p, pre, own, Q)
    for s in range(0, n_seq, max(1, n_seq // 10)):
        K, V, w = (torch.cat([a[s % n_pre], b[s]]) for a, b in zip(pre, own))
        _check_out(out[s], lse[s], _attention(Q[s].reshape(-1, d), K, V, w), dtype, cp + cs, "sequence %d" % s)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_seq,nq,first", [(2, 30, 55), (2, 190, -25), (2, 100, 40), (200, 100, 40), (200, 130, 20)])
def test_an_infinite_weight_reaches_those_that_see_it(bk, dtype, n_seq, nq, first):  # noqa: F811
    """inf / inf for every query that sees the token, nothing for the others, also where a whole tile weighs that much."""
    gen, d = _gen(nq), 128
    K, V, w = _cache(gen, n_seq, 200, d, dtype, absent=0.1, poison=False)
    Q = torch.randn(n_seq, 1, nq, d, generator=gen, device="cuda").to(dtype)
    p = bk.make_params(d, 64, 1, dtype, log_c=0.0)
    ref, lse, _ = bk.attend_mass(p, K, V, w, Q, visible=first)
    w[:, 64:128] = float("inf")
    out, lse2, _ = bk.attend_mass(p, K, V, w, Q, visible=first)
    before = 64 - first + 1                                      # queries that see 64 places at most
    assert 0 < before < nq
    assert torch.equal(out[:, :, :before], ref[:, :, :before]) and torch.equal(lse[:, :, :before], lse2[:, :, :before])
    assert bool(out[:, :, before:].isnan().all()) and bool(lse2[:, :, before:].isnan().all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_seq,count,g,nq", [(2, 200, 4, 1), (2, 3000, 4, 1), (200, 2000, 4, 1), (2, 200, 4, 30), (2, 3000, 4, 30), (300, 50, 1, 17)])
def test_a_query_of_nan(bk, dtype, n_seq, count, g, nq):  # noqa: F811
    """Its answer, its lse and the masses of its sequence's tokens are NaN; places without a token, other queries and sequences stay as they are."""
    gen, d = _gen(count), 128
    K, V, w = _cache(gen, n_seq, count, d, dtype)
    Q = torch.randn(n_seq, g, nq, d, generator=gen, device="cuda").to(dtype)
    p = bk.make_params(d, 64, 1, dtype, log_c=0.0)
    ref = bk.attend_mass(p, K, V, w, Q)
    z, l = bk.attend_prefix(p, (K[:1], V[:1], w[:1]), (K, V, w), Q)
    Q[1, g - 1, nq - 1, 5] = float("nan")
    got = bk.attend_mass(p, K, V, w, Q)
    z2, l2 = bk.attend_prefix(p, (K[:1], V[:1], w[:1]), (K, V, w), Q)
    for (o, x), (o2, x2) in (((ref[0], ref[1]), (got[0], got[1])), ((z, l), (z2, l2))):
        assert bool(o2[1, g - 1, nq - 1].isnan().all()) and bool(x2[1, g - 1, nq - 1].isnan())
        o2[1, g - 1, nq - 1], x2[1, g - 1, nq - 1] = o[1, g - 1, nq - 1], x[1, g - 1, nq - 1]
        assert torch.equal(o, o2) and torch.equal(x, x2)
    live = w[1] > 0
    assert bool(got[2][1][live].isnan().all()) and bool((got[2][1][~live] == 0).all())
    got[2][1] = ref[2][1]
    assert torch.equal(got[2], ref[2])


WHOLE = [  # dtype, d, n_seq, count, g, nq: sequences whose logits one workgroup holds (11 sixteenths of the compute units or more), up to what LDS takes and past it
    (BF16, 128, 176, 2001, 4, 1), (F32, 128, 180, 777, 16, 1), (F32, 64, 177, 1001, 1, 1), (BF16, 128, 176, 8768, 4, 1), (BF16, 128, 176, 9152, 4, 1),
    (BF16, 128, 176, 9153, 4, 1), (F32, 128, 180, 1488, 16, 1), (F32, 128, 180, 1489, 16, 1), (BF16, 64, 200, 4480, 8, 1), (BF16, 128, 520, 4576, 4, 1),
    (BF16, 128, 520, 4577, 4, 1), (F32, 64, 176, 20320, 1, 2),
]


def _whole(bk, dtype, d, n_seq, count, g, nq):  # noqa: F811
    gen = _gen(count + n_seq)
    K, V, w = _cache(gen, n_seq, count, d, dtype)
    Q = (2.0 * torch.randn(n_seq, g, nq, d, generator=gen, device="cuda")).to(dtype)
    return K, V, w, Q, torch.rand(n_seq, count, generator=gen, device="cuda"), bk.make_params(d, 64, 1, dtype, log_c=0.0)


@pytest.mark.parametrize("dtype,d,n_seq,count,g,nq", WHOLE)
def test_mass_of_whole_sequences(bk, dtype, d, n_seq, count, g, nq):  # noqa: F811
    K, V, w, Q, before, p = _whole(bk, dtype, d, n_seq, count, g, nq)
    out, lse, mass = bk.attend_mass(p, K, V, w, Q, before, decay=0.5)
    for s in range(0, n_seq, n_seq // 8):
        ref = _attention(Q[s].reshape(-1, d), K[s], V[s], w[s])
        _check_out(out[s], lse[s], ref, dtype, count, "sequence %d" % s)
        _check_mass(mass[s], before[s], 0.5, ref, count, g * nq, "sequence %d" % s)


@pytest.mark.parametrize("count", [9152, 9153])
def test_the_longest_whole_sequences_captured(bk, count):  # noqa: F811
    K, V, w, Q, before, p = _whole(bk, BF16, 128, 176, count, 4, 1)
    ws = torch.empty(bk.attend_mass_workspace_bytes(p, 176, count, 4, 1), device="cuda", dtype=torch.uint8)
    step = lambda: bk.attend_mass(p, K, V, w, Q, before, decay=0.5, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for turn in range(3):
        want = [t.clone() for t in step()]
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), turn
        Q.mul_(0.9)
        before.add_(0.125)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("g,nq", [(2, 1), (4, 12), (2, 64)])
def test_sequences_of_different_lengths_that_end_together(bk, dtype, g, nq):  # noqa: F811
    """Empty places in front: the last nq tokens of every sequence see what lies before them, and a recent window holds last tokens."""
    gen, n_seq, count, d = _gen(nq), 6, 500, 128
    K, V, w = _cache(gen, n_seq, count, d, dtype, absent=0.0)
    length = [500, 437, 64, 65, 1, 0]
    for s, n in enumerate(length):
        w[s, :count - n], K[s, :count - n], V[s, :count - n] = 0.0, float("nan"), float("inf")
    Q = torch.randn(n_seq, g, nq, d, generator=gen, device="cuda").to(dtype)
    p = bk.make_params(d, 64, 1, dtype, log_c=0.0)
    out, lse, mass = bk.attend_mass(p, K, V, w, Q, visible=count - nq + 1)
    kept = bk.evict(p, K, V, w, mass, 70, n_recent=20)
    for s, n in enumerate(length):
        own = slice(count - n, count)
        sees = (n - nq + 1 + torch.arange(nq, device="cuda")).repeat(g)
        ref = _attention(Q[s].reshape(-1, d), K[s, own], V[s, own], w[s, own], sees)
        _check_out(out[s], lse[s], ref, dtype, count, "sequence %d" % s)
        assert bool((mass[s, :count - n] == 0).all())
        if n:
            _check_mass(mass[s, own], mass[s, own], 0.0, ref, n, g * nq, "sequence %d" % s)
        stay = min(n, 70)
        assert int(kept["count"][s]) == stay
        idx = kept["idx"][s, :stay].tolist()
        assert idx == sorted(idx) and set(range(count - min(n, 20), count)) <= set(idx) <= set(range(count - n, count))
        others = mass[s, own][:max(n - 20, 0)].sort(descending=True).values[:max(stay - 20, 0)]
        assert torch.equal(kept["mass"][s, :max(stay - 20, 0)].sort(descending=True).values, others)


@pytest.mark.parametrize("count,keep", [(900, 100), (70000, 5000)])
def test_windows_of_sequences_that_begin_together(bk, count, keep):  # noqa: F811
    """Empty places behind: a mass of +inf keeps a token before all others, so every sequence has windows at its own ends."""
    gen, n_seq, d = _gen(count), 4, 64
    K, V, w = _cache(gen, n_seq, count, d, BF16, absent=0.0)
    mass = torch.rand(n_seq, count, generator=gen, device="cuda")
    length = [count, count // 2 + 1, 40, 0]
    marked = mass.clone()
    for s, n in enumerate(length):
        w[s, n:] = 0.0
        marked[s, :min(n, 4)] = math.inf
        marked[s, max(n - 30, 0):n] = math.inf
    kept = bk.evict(bk.make_params(d, 64, 1, BF16, log_c=0.0), K, V, w, marked, keep)
    for s, n in enumerate(length):
        stay = min(n, keep)
        assert int(kept["count"][s]) == stay
        idx = kept["idx"][s, :stay].tolist()
        window = set(range(min(n, 4))) | set(range(max(n - 30, 0), n))
        assert idx == sorted(idx) and window <= set(idx) <= set(range(n))
        rest = sorted(set(idx) - window)
        outside = sorted(set(range(n)) - window)
        want = mass[s][outside].sort(descending=True).values[:len(rest)] if outside else mass[s, :0]
        assert torch.equal(mass[s][rest].sort(descending=True).values if rest else mass[s, :0], want)


@pytest.mark.parametrize("dtype,d,n_seq,count,keep", [(BF16, 64, 2, 32768, 9000), (BF16, 128, 1, 32769, 5), (F32, 64, 2, 50001, 50001), (BF16, 64, 3, 65536, 65535),
                                                      (F32, 128, 1, 65536, 16384), (BF16, 64, 2, 65537, 16384), (BF16, 128, 2, 131072, 32768)])
@pytest.mark.parametrize("masses", ["spread", "ties", "equal"])
def test_evict_from_long_sequences(bk, dtype, d, n_seq, count, keep, masses):  # noqa: F811
    """Both sides of what one workgroup has registers for."""
    gen = _gen(count + keep)
    K, V, w = _cache(gen, n_seq, count, d, dtype, absent=0.05)
    mass = torch.exp(2.0 * torch.randn(n_seq, count, generator=gen, device="cuda"))
    if masses == "ties":
        mass = torch.floor(5.0 * torch.rand(n_seq, count, generator=gen, device="cuda"))
    elif masses == "equal":
        mass = torch.full_like(mass, 0.25)
    sink, recent = min(4, keep), min(100, keep - min(4, keep))
    res = bk.evict(bk.make_params(d, 64, 1, dtype, log_c=0.0), K, V, w, mass, keep, n_sink=sink, n_recent=recent)
    _check_evict(res, K, V, w, mass, None, count, keep, sink, recent)


def test_launches_of_evict_are_recorded(bk):  # noqa: F811
    """Few rows: one launch.  Many: search and copy.  Long sequences: three counts, two passes for the list, and the copy."""
    from paper_2502_07861_amd import binding
    p = bk.make_params(64, 64, 1, BF16, log_c=0.0)
    gen = _gen(2)
    for n_seq, count, keep, want in ((3, 500, 100, [4]), (2, 9000, 4000, [4, 5]), (1, 70000, 3000, [4, 4, 4, 4, 4, 5])):
        K, V, w = _cache(gen, n_seq, count, 64, BF16)
        mass = torch.rand(n_seq, count, generator=gen, device="cuda")
        binding.profile_enable(16)
        try:
            bk.evict(p, K, V, w, mass, keep)
            records = binding.profile_read(16)
        finally:
            binding.profile_enable(0)
        assert [k for k, _, _ in records] == want
        assert all(ms > 0 for _, ms, _ in records)
        assert [u for _, _, u in records] == [n_seq * (count if k == 4 else keep) for k in want]
