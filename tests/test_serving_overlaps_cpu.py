"""attend_prefix, attend_mass and evict refuse outputs that lie on what they read or on each other: host-side checks, addresses that are never
dereferenced.  What lies between is let through to the workspace's check, which refuses it."""
import ctypes as C
import random

import pytest

from test_serving_cpu import AT, _evict, bk  # noqa: F401  (bk: a fixture)


def _prefix(bk, p, n_pre=2, count_p=100, stride_p=100, n_seq=6, count_s=10, stride_s=10, g=2, nq=1, K_p=AT[0], V_p=AT[1], w_p=AT[2],  # noqa: F811
            K_s=AT[3], V_s=AT[4], w_s=AT[5], Q=AT[6], out=AT[7], lse=AT[9]):
    return bk.lib().bkv_attend_prefix(C.byref(p), K_p, V_p, w_p, n_pre, count_p, stride_p, K_s, V_s, w_s, n_seq, count_s, stride_s, Q, g, nq, out, lse,
                                      None, 0, None)


def _mass(bk, p, n_seq=2, count=100, stride=128, g=2, nq=3, visible=100, decay=1.0, K=AT[0], V=AT[1], w=AT[2], Q=AT[3], mass=AT[4], out=AT[5],  # noqa: F811
          mass_out=AT[6], lse=AT[7]):
    return bk.lib().bkv_attend_mass(C.byref(p), K, V, w, n_seq, count, stride, Q, g, nq, visible, decay, mass, out, lse, mass_out, None, 0, None)


def test_prefix(bk):  # noqa: F811
    p = bk.make_params(128, 64, 1, bk.BKV_BF16, log_c=0.0)                # rows of 256 bytes
    assert _prefix(bk, p) == bk.BKV_EWORKSPACE
    for at in range(7):                                                   # the last bytes of every input, and its first
        last = [2 * 100 * 256, 2 * 100 * 256, 2 * 100 * 4, 60 * 256, 60 * 256, 60 * 4, 12 * 256][at]
        for lo in (AT[at], AT[at] + last - 16):
            assert _prefix(bk, p, out=lo) == bk.BKV_EINVAL, at
            assert _prefix(bk, p, lse=lo) == bk.BKV_EINVAL, at
        assert _prefix(bk, p, out=AT[at] + last) == bk.BKV_EWORKSPACE, at
        assert _prefix(bk, p, lse=AT[at] - 12 * 4) == bk.BKV_EWORKSPACE, at
    assert _prefix(bk, p, lse=AT[7] + 12 * 256 - 4) == bk.BKV_EINVAL and _prefix(bk, p, lse=AT[7] + 12 * 256) == bk.BKV_EWORKSPACE
    assert _prefix(bk, p, out=AT[3], count_s=0) == bk.BKV_EWORKSPACE       # not read
    # between two prefixes' places: 50 of 100 are read
    assert _prefix(bk, p, out=AT[0] + 50 * 256, count_p=50) == bk.BKV_EWORKSPACE
    assert _prefix(bk, p, out=AT[0] + 89 * 256, count_p=50) == bk.BKV_EINVAL


def test_mass(bk):  # noqa: F811
    p = bk.make_params(64, 64, 1, bk.BKV_F32, log_c=0.0)                  # rows of 256 bytes, 100 places of 128
    assert _mass(bk, p) == bk.BKV_EWORKSPACE
    for name in ("out", "lse", "mass_out"):
        for at, elem in ((0, 256), (1, 256), (2, 4)):
            for lo in (AT[at], AT[at] + 99 * elem // 16 * 16, AT[at] + 128 * elem, AT[at] + (128 + 99) * elem // 16 * 16):
                assert _mass(bk, p, **{name: lo}) == bk.BKV_EINVAL, (name, at)
        assert _mass(bk, p, **{name: AT[3] + 11 * 256}) == bk.BKV_EINVAL and _mass(bk, p, **{name: AT[3] + 12 * 256}) == bk.BKV_EWORKSPACE
    assert _mass(bk, p, lse=AT[0] + 100 * 256) == bk.BKV_EWORKSPACE        # between the sequences
    assert _mass(bk, p, out=AT[0] + (128 + 100) * 256) == bk.BKV_EWORKSPACE
    for k in (dict(lse=AT[5]), dict(mass_out=AT[5]), dict(mass_out=AT[7]), dict(lse=AT[6] + 99 * 4), dict(out=AT[4]), dict(lse=AT[4]), dict(mass_out=AT[4] + 4),
              dict(mass_out=AT[4] + 128 * 4), dict(mass_out=AT[4] - 4), dict(out=AT[6], mass=AT[6])):
        assert _mass(bk, p, **k) == bk.BKV_EINVAL, k
    assert _mass(bk, p, mass_out=AT[4]) == bk.BKV_EWORKSPACE               # in place
    # two arrays a sequence in one buffer, one behind the other
    assert _mass(bk, p, stride=256, mass_out=AT[2] + 128 * 4) == bk.BKV_EWORKSPACE
    assert _mass(bk, p, stride=256, mass_out=AT[2] + 99 * 4) == bk.BKV_EINVAL
    assert _mass(bk, p, stride=256, mass_out=AT[2] + 157 * 4) == bk.BKV_EINVAL


def test_evict(bk):  # noqa: F811
    p = bk.make_params(64, 64, 1, bk.BKV_BF16, log_c=0.0)                 # rows of 128 bytes, 100 places of 128
    no = lambda **k: _evict(bk, p, **k)
    assert no(ws=None) == bk.BKV_EWORKSPACE
    assert no(w_out=AT[2] + 100 * 4, ws=None, keep=5, recent=1) == bk.BKV_EWORKSPACE          # 10 numbers in a gap of 28
    assert no(w_out=AT[2] + 100 * 4, ws=None) == bk.BKV_EINVAL                                # 80 of them
    assert no(w_out=AT[2] + 228 * 4, ws=None) == bk.BKV_EWORKSPACE
    assert no(count_out=AT[0] + 100 * 128, ws=None) == bk.BKV_EWORKSPACE and no(count_out=AT[0] + 100 * 128 - 4) == bk.BKV_EINVAL


@pytest.mark.parametrize("seed", range(4))
def test_every_place(bk, seed):  # noqa: F811
    """mass_out against w, both in pieces, at many distances, against sets of places."""
    rng = random.Random(seed)
    p = bk.make_params(64, 64, 1, bk.BKV_F32, log_c=0.0)
    for _ in range(200):
        n, count = rng.randrange(1, 6), rng.randrange(1, 9)
        stride = count + rng.choice([0, 1, 3, 10])
        off = rng.randrange(-n * stride - 10, n * stride + 10)
        a = {i * stride + k for i in range(n) for k in range(count)}
        meet = bool(a & {x + off for x in a})
        # the whole of K, V lies elsewhere
        got = _mass(bk, p, n_seq=n, count=count, stride=stride, visible=count, w=AT[2] + 4096, mass_out=AT[2] + 4096 + 4 * off)
        assert got == (bk.BKV_EINVAL if meet else bk.BKV_EWORKSPACE), (n, count, stride, off)


def test_one_sequence_may_name_any_stride(bk):  # noqa: F811
    p = bk.make_params(64, 64, 1, bk.BKV_F32, log_c=0.0)
    for stride in (100, 2**56, 2**62, 2**63 - 1):                          # bytes past 64 bits
        assert _mass(bk, p, n_seq=1, stride=stride) == bk.BKV_EWORKSPACE
        assert _mass(bk, p, n_seq=1, stride=stride, out=AT[0] + 99 * 256) == bk.BKV_EINVAL
        assert _mass(bk, p, n_seq=1, stride=stride, lse=AT[0] + 100 * 256) == bk.BKV_EWORKSPACE
        assert _mass(bk, p, n_seq=1, stride=stride, mass_out=AT[4] + 4) == bk.BKV_EINVAL
        assert _evict(bk, p, n_seq=1, stride=stride, ws=None) == bk.BKV_EWORKSPACE
