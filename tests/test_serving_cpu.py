"""What attend_prefix, attend_mass and evict refuse, and what their workspaces hold: host-side checks that end before any launch."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def bk():
    import os
    from paper_2502_07861_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2502_07861_amd.build import build
        build()
    binding.lib()
    return binding


AT = [0x100000 * (i + 1) for i in range(16)]         # addresses that are never dereferenced, 1 MiB apart


def _prefix(bk, p, n_pre=2, count_p=100, stride_p=100, n_seq=6, count_s=10, stride_s=10, g=2, nq=1, K_p=AT[0], V_p=AT[1], w_p=AT[2], K_s=AT[3],
            V_s=AT[4], w_s=AT[5], Q=AT[6], out=AT[7], ws=AT[8], ws_bytes=1 << 30):
    return bk.lib().bkv_attend_prefix(C.byref(p) if p else None, K_p, V_p, w_p, n_pre, count_p, stride_p, K_s, V_s, w_s, n_seq, count_s, stride_s, Q, g,
                                      nq, out, None, ws, ws_bytes, None)


def _mass(bk, p, n_seq=2, count=100, stride=128, g=2, nq=3, visible=100, decay=1.0, K=AT[0], V=AT[1], w=AT[2], Q=AT[3], mass=AT[4], out=AT[5],
          mass_out=AT[6], ws=AT[8], ws_bytes=1 << 30):
    return bk.lib().bkv_attend_mass(C.byref(p) if p else None, K, V, w, n_seq, count, stride, Q, g, nq, visible, decay, mass, out, None, mass_out, ws,
                                    ws_bytes, None)


def _evict(bk, p, n_seq=2, count=100, stride=128, keep=40, sink=4, recent=8, K=AT[0], V=AT[1], w=AT[2], mass=AT[3], idx=None, K_out=AT[4],
           V_out=AT[5], w_out=AT[6], mass_out=AT[7], idx_out=AT[9], count_out=AT[10], ws=AT[8], ws_bytes=1 << 30):
    return bk.lib().bkv_evict(C.byref(p) if p else None, K, V, w, mass, idx, n_seq, count, stride, keep, sink, recent, K_out, V_out, w_out, mass_out,
                              idx_out, count_out, ws, ws_bytes, None)


def test_prefix_refusals(bk):
    p = bk.make_params(128, 64, 1, bk.BKV_BF16, log_c=0.0)
    no = lambda **k: _prefix(bk, p, **k)
    assert _prefix(bk, None) == bk.BKV_EINVAL
    assert _prefix(bk, bk.make_params(96, 64, 1, bk.BKV_BF16, log_c=0.0)) == bk.BKV_ESHAPE
    for k in (dict(n_pre=0), dict(n_pre=-2), dict(n_pre=4), dict(n_seq=-6), dict(n_seq=7), dict(count_p=-1), dict(count_p=101), dict(count_s=-1),
              dict(count_s=11), dict(g=0), dict(nq=0), dict(K_p=None), dict(V_p=None), dict(w_p=None), dict(K_s=None), dict(V_s=None), dict(w_s=None),
              dict(Q=None), dict(out=None), dict(K_p=AT[0] + 8), dict(V_s=AT[4] + 8), dict(Q=AT[6] + 4), dict(out=AT[7] + 2), dict(out=AT[6]),
              dict(out=AT[6] + 256)):
        assert no(**k) == bk.BKV_EINVAL, k
    for k in (dict(n_seq=65536, n_pre=1), dict(g=4, nq=65536), dict(n_seq=60000, g=4, nq=60000), dict(count_p=2**31, stride_p=2**31),
              dict(count_s=2**31, stride_s=2**31)):
        assert no(**k) == bk.BKV_ESHAPE, k
    for k in (dict(ws=None), dict(ws_bytes=16), dict(ws=AT[8] + 8)):
        assert no(**k) == bk.BKV_EWORKSPACE, k
    assert no(n_seq=0) == bk.BKV_OK


def test_mass_refusals(bk):
    p = bk.make_params(64, 64, 1, bk.BKV_F32, log_c=0.0)
    no = lambda **k: _mass(bk, p, **k)
    assert _mass(bk, None) == bk.BKV_EINVAL
    assert _mass(bk, bk.make_params(64, 64, 1, 5, log_c=0.0)) == bk.BKV_ESHAPE
    for k in (dict(n_seq=-1), dict(count=-1), dict(count=129), dict(g=0), dict(nq=-1), dict(decay=-0.1), dict(decay=1.1), dict(decay=float("nan")),
              dict(K=None), dict(V=None), dict(w=None), dict(Q=None), dict(out=None), dict(mass_out=None), dict(K=AT[0] + 4), dict(V=AT[1] + 8),
              dict(Q=AT[3] + 8), dict(out=AT[5] + 8), dict(out=AT[3]), dict(mass_out=AT[4] + 128), dict(mass_out=AT[2]), dict(mass_out=AT[2] + 256)):
        assert no(**k) == bk.BKV_EINVAL, k
    for k in (dict(n_seq=65536), dict(g=4, nq=65536), dict(n_seq=60000, g=4, nq=60000), dict(count=2**31, stride=2**31)):
        assert no(**k) == bk.BKV_ESHAPE, k
    for k in (dict(ws=None), dict(ws_bytes=16), dict(ws=AT[8] + 8)):
        assert no(**k) == bk.BKV_EWORKSPACE, k
    assert no(n_seq=0) == bk.BKV_OK


def test_evict_refusals(bk):
    p = bk.make_params(64, 64, 1, bk.BKV_BF16, log_c=0.0)
    no = lambda **k: _evict(bk, p, **k)
    assert _evict(bk, None) == bk.BKV_EINVAL
    for k in (dict(n_seq=-1), dict(count=-1), dict(count=129), dict(keep=-1), dict(keep=101), dict(sink=-1), dict(recent=-1), dict(sink=33),
              dict(sink=2**62, recent=2**62), dict(recent=37), dict(K=None), dict(V=None), dict(w=None), dict(mass=None), dict(K_out=None),
              dict(V_out=None), dict(K=AT[0] + 8), dict(V=AT[1] + 4), dict(K_out=AT[4] + 8), dict(V_out=AT[5] + 2), dict(K_out=AT[0]),
              dict(V_out=AT[0] + 128), dict(V_out=AT[1] + 128 * 40), dict(K_out=AT[5]), dict(w_out=AT[2]), dict(mass_out=AT[3] + 4), dict(w_out=AT[6], mass_out=AT[6]),
              dict(idx=AT[11], idx_out=AT[11]), dict(count_out=AT[9])):
        assert no(**k) == bk.BKV_EINVAL, k
    for k in (dict(n_seq=65536), dict(count=2**31, stride=2**31)):
        assert no(**k) == bk.BKV_ESHAPE, k
    for k in (dict(ws=None), dict(ws_bytes=16), dict(ws=AT[8] + 8)):
        assert no(**k) == bk.BKV_EWORKSPACE, k
    assert no(n_seq=0) == bk.BKV_OK
    assert no(keep=0, sink=0, recent=0, count_out=None) == bk.BKV_OK                # nothing to write


def test_workspaces(bk):
    """0 for what the calls refuse; enough for the partial rows of every split (d + 4 floats a query) else, whatever the counts."""
    L = bk.lib()
    p = bk.make_params(128, 64, 1, bk.BKV_BF16, log_c=0.0)
    pre = lambda *a: bk.attend_prefix_workspace_bytes(p, *a)
    assert pre(3, 7, 4, 1) == 0 and pre(0, 4, 4, 1) == 0 and pre(1, 4, 0, 1) == 0 and pre(1, 65536, 1, 1) == 0
    assert pre(2, 8, 4, 1) >= 2 * 8 * 4 * 132 * 4
    mass = lambda *a: bk.attend_mass_workspace_bytes(p, *a)
    assert mass(2, -1, 4, 1) == 0 and mass(2, 10, 4, 0) == 0
    assert mass(2, 100, 4, 1) >= 2 * 4 * 8
    assert all(mass(3, c, 4, 5) <= mass(3, 1 << 20, 4, 5) for c in (0, 1, 1000, 99999))
    ev = lambda *a: bk.evict_workspace_bytes(p, *a)
    assert ev(-1, 10) == 0 and ev(2, -1) == 0 and ev(2, 100) >= 2 * 100 * 4 and L.bkv_evict_workspace_bytes(None, 2, 100) == 0


def test_binding_refuses_before_the_library(bk):
    """Shapes, devices: ValueError from the binding, with host tensors that never reach the library."""
    p = bk.make_params(64, 64, 1, torch.float32, log_c=0.0)
    K, V, w = torch.zeros(4, 10, 64), torch.zeros(4, 10, 64), torch.zeros(4, 10)
    Q = torch.zeros(4, 2, 1, 64)
    for call in (lambda: bk.attend_prefix(p, (K, V, w), (K, V, w), Q),                                       # not on the GPU
                 lambda: bk.attend_prefix(p, (K, V, w[:, :9]), (K, V, w), Q),
                 lambda: bk.attend_prefix(p, (K, V, w), (K, V[:3], w), Q),
                 lambda: bk.attend_prefix(p, (K, V, w), (K, V, w), Q[:3]),
                 lambda: bk.attend_mass(p, K, V, w, Q),
                 lambda: bk.attend_mass(p, K, V, w, Q, w[:, :9]),
                 lambda: bk.attend_mass(p, K[:, :, :32], V, w, Q),
                 lambda: bk.evict(p, K, V, w, w, 5),
                 lambda: bk.evict(p, K, V, w, w[:3], 5),
                 lambda: bk.evict(p, K, V, w, w, 11)):
        with pytest.raises(ValueError):
            call()
