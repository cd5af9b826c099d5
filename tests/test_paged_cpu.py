"""The paged cache without a GPU: its oracle against textbook forms, the binding's
shape checks, and the library's refusals (all before anything is launched)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_18410_amd as rs
from oracle import paged as O

bf, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


# ---- oracle --------------------------------------------------------------

def _np_cache(n, H, P, dh, G, vcap):
    return dict(K=np.zeros((n, H, P, dh)), V=np.zeros((n, H, vcap, dh // G)), mask=np.zeros((n, P), np.uint32),
                slot=np.zeros((n, P), np.int32))


def test_oracle_append_then_attend_is_dense_attention():
    rng = np.random.default_rng(0)
    B, H, rep, dh, G, P, T = 2, 2, 3, 16, 4, 16, 37
    c = _np_cache(6, H, P, dh, G, P * G)
    table = rng.permutation(6).reshape(2, 3)
    k, z = rng.standard_normal((2, B, T, H, dh))
    mask = rng.integers(0, 16, (B, T))
    for lo, hi in ((0, 5), (5, 16), (16, 17), (17, 37)):
        O.append(c, k[:, lo:hi], z[:, lo:hi], mask[:, lo:hi], table, [lo] * B)
    q = rng.standard_normal((B, 2, H * rep, dh))
    R = np.linalg.qr(rng.standard_normal((H, dh, dh)))[0]
    vis = np.array([[37, 20], [0, 1]])
    out, w, _, _ = O.attend(q, c, table, [37, 37], R, visible=vis, mass=np.ones((B, 48)), decay=0.5)
    for b in range(B):
        zz = z[b].reshape(T, H, G, -1) * ((mask[b][:, None] >> np.arange(G)) & 1)[:, None, :, None]
        p_all = np.zeros(T)
        for j in range(2):
            n = vis[b, j]
            for h in range(H * rep):
                if n == 0:
                    assert not out[b, j, h].any()
                    continue
                s = k[b, :n, h // rep] @ q[b, j, h] / 4.0
                p = np.exp(s) / np.exp(s).sum()
                p_all[:n] += p
                np.testing.assert_allclose(out[b, j, h], R[h // rep] @ (p @ zz[:n, h // rep].reshape(n, dh)), atol=1e-12)
        np.testing.assert_allclose(w[b, :T], 0.5 + p_all, atol=1e-12)
        assert (w[b, T:] == 1).all()


def test_oracle_evict_and_compact():
    rng = np.random.default_rng(1)
    mass = np.array([[5, 1, np.nan, 3, 3, -0.0, 0.0, 9, 2]], dtype=np.float32)
    idx, n = O.evict(mass, [9], 5, first=1, recent=2)
    assert idx.tolist() == [[0, 3, 4, 7, 8]] and n.tolist() == [5]
    idx, n = O.evict(mass, [9], 8, first=0, recent=0)
    assert idx.tolist() == [[0, 1, 3, 4, 5, 6, 7, 8]]
    idx, n = O.evict(mass, [3], 5)
    assert idx.tolist() == [[0, 1, 2, -1, -1]] and n.tolist() == [3]
    src, dst = _np_cache(4, 1, 16, 8, 4, 64), _np_cache(3, 1, 16, 8, 4, 64)
    k, z = rng.standard_normal((2, 1, 50, 1, 8))
    mask = rng.integers(0, 16, (1, 50))
    O.append(src, k, z, mask, np.array([[2, 0, 3, 1]]), [0])
    keep = np.sort(rng.permutation(50)[:20])[None]
    O.compact(src, np.array([[2, 0, 3, 1]]), keep, [20], dst, np.array([[1, 2]]))
    again = _np_cache(3, 1, 16, 8, 4, 64)
    O.append(again, k[:, keep[0]], z[:, keep[0]], mask[:, keep[0]], np.array([[1, 2]]), [0])
    for x in dst:
        assert np.array_equal(dst[x], again[x]), x


def test_oracle_rotary_is_a_rotation():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((1, 3, 2, 16))
    pos = rng.integers(0, 1000, (1, 3, 2))
    f, ax = 10000.0 ** (-np.arange(6) / 6), np.array([0, 1, 0, 1, 1, 5])
    for il in (False, True):
        y = O.rotary(x, pos, f, ax, il)
        np.testing.assert_allclose(O.rotary(y, pos, f, ax, il, inverse=True), x, atol=1e-13)
        assert np.array_equal(y[..., 12:], x[..., 12:])
        p, q = (10, 11) if il else (5, 11)
        assert np.array_equal(y[..., p], x[..., p]) and np.array_equal(y[..., q], x[..., q])  # axis 5 of 2: not turned
        z = x[..., 0] + 1j * x[..., 1 if il else 6]
        w = z * np.exp(1j * pos[:, :, 0] * 1.0)[:, :, None]
        np.testing.assert_allclose(y[..., 0], w.real, atol=1e-13)
        np.testing.assert_allclose(y[..., 1 if il else 6], w.imag, atol=1e-13)


# ---- binding -------------------------------------------------------------

B, T, H, Hq, dh, G, P, N, W = 2, 3, 2, 4, 64, 8, 16, 5, 2


def z(*shape, dtype=bf):
    return torch.zeros(shape, dtype=dtype)


def cache(**kw):
    c = dict(K=z(N, H, P, dh), V=z(N, H, P * 4, dh // G), mask=z(N, P, dtype=i32), slot=z(N, P, dtype=i32))
    c.update(kw)
    return rs.PagedCache(**c)


def reaches_device_check(fn, *a, **kw):
    with pytest.raises(ValueError, match="device tensors only"):
        fn(*a, **kw)


def refused(fn, *a, match="expected (shape|dtype)", **kw):
    with pytest.raises((ValueError, TypeError), match=match):
        fn(*a, **kw)


def test_rotary_shapes():
    q, k = z(B, T, Hq, dh), z(B, T, H, dh)
    pos, f, ax = z(B, T, 3, dtype=i32), z(32, dtype=f32), z(32, dtype=u8)
    reaches_device_check(rs.rotary, q, k, pos, f, ax)
    reaches_device_check(rs.rotary, None, k, pos[..., 0], f)
    refused(rs.rotary, q, k[:1], pos, f, ax)
    refused(rs.rotary, q, k.float(), pos, f, ax)
    refused(rs.rotary, q, k, pos.long(), f, ax)
    refused(rs.rotary, q, k, pos[:, :2], f, ax)
    refused(rs.rotary, q, k, pos, f.double(), ax)
    refused(rs.rotary, q, k, pos, f, ax[:5])
    refused(rs.rotary, None, None, pos, f, match="both None")


@pytest.mark.parametrize("bad", [
    dict(V=z(N, H, 8, 7)), dict(V=z(N, H + 1, 8, 8)), dict(V=z(N, H, 8, 8, dtype=f32)), dict(mask=z(N, P + 1, dtype=i32)),
    dict(slot=z(N, P)), dict(K=z(N, H, P, dh, dtype=torch.float16)),
])
def test_cache_shapes(bad):
    a = (z(B, T, H, dh), z(B, T, H, dh), z(B, T, dtype=i32), z(B, W, dtype=i32), z(B, dtype=i32))
    with pytest.raises((ValueError, TypeError)):
        rs.cache_append(cache(**bad), *a)
    with pytest.raises((ValueError, TypeError)):
        rs.attend_paged(z(B, T, Hq, dh), cache(**bad), a[3], a[4])


def test_append_shapes():
    k, zz, m, t, n = z(B, T, H, dh), z(B, T, H, dh), z(B, T, dtype=i32), z(B, W, dtype=i32), z(B, dtype=i32)
    reaches_device_check(rs.cache_append, cache(), k, zz, m, t, n)
    refused(rs.cache_append, cache(), z(B, T, Hq, dh), zz, m, t, n)
    refused(rs.cache_append, cache(), k.float(), zz, m, t, n)
    refused(rs.cache_append, cache(), k, zz, m[:, :2], t, n)
    refused(rs.cache_append, cache(), k, zz, m, t.long(), n)
    refused(rs.cache_append, cache(), k, zz, m, t[:1], n)
    refused(rs.cache_append, cache(), k, zz, m, t, n[:1])
    refused(rs.cache_append, cache(), k, zz, m, t, n, n_new=n.long())


def test_attend_paged_shapes():
    q, t, n = z(B, T, Hq, dh), z(B, W, dtype=i32), z(B, dtype=i32)
    reaches_device_check(rs.attend_paged, q, cache(), t, n)
    refused(rs.attend_paged, z(B, T, Hq, 2 * dh), cache(), t, n)
    refused(rs.attend_paged, q.float(), cache(), t, n)
    refused(rs.attend_paged, q, cache(), t, n.long())
    refused(rs.attend_paged, q, cache(), t, n, R=z(Hq, dh, dh))
    refused(rs.attend_paged, q, cache(), t, n, visible=z(B, T + 1, dtype=i32))
    refused(rs.attend_paged, q, cache(), t, n, mass=z(B + 1, 9, dtype=f32))
    refused(rs.attend_paged, q, cache(), t, n, mass=z(B, 40, dtype=f32), mass_out=z(B, 41, dtype=f32))
    refused(rs.attend_paged, q, cache(), t, n, out=z(B, T, H, dh))
    refused(rs.attend_paged, q, cache(), t, n, workspace=z(8, dtype=f32))


def test_evict_and_compact_shapes():
    m, n = z(B, 40, dtype=f32), z(B, dtype=i32)
    reaches_device_check(rs.evict_tokens, m, n, 8)
    refused(rs.evict_tokens, m.double(), n, 8)
    refused(rs.evict_tokens, m, n[:1], 8)
    refused(rs.evict_tokens, m, n, 0, match="at least 1")
    refused(rs.evict_tokens, m, n, 8, out=(z(B, 9, dtype=i32), n))
    t, idx = z(B, W, dtype=i32), z(B, 8, dtype=i32)
    reaches_device_check(rs.cache_compact, cache(), t, idx, n, cache(), t)
    refused(rs.cache_compact, cache(), t, idx.long(), n, cache(), t)
    refused(rs.cache_compact, cache(), t, idx, n[:1], cache(), t)
    refused(rs.cache_compact, cache(), t[:1], idx, n, cache(), t)
    refused(rs.cache_compact, cache(), t, idx, n, cache(), t, mass_out=m, match="without mass")
    refused(rs.cache_compact, cache(), t, idx, n, cache(K=z(N, H, P, dh, dtype=f32), V=z(N, H, 8, 8, dtype=f32)), t)


# ---- C ABI ---------------------------------------------------------------

A0, A1, A2, A3 = (ctypes.c_void_p(x) for x in (0x10000000, 0x20000000, 0x30000000, 0x40000000))  # never dereferenced


@pytest.fixture(scope="module")
def lib():
    return rs.load()


def _last():
    return rs.load().rolesub_last_error().decode()


def _pages(**kw):
    d = dict(n_pages=5, page=16, vcap=64, H=2, dh=64, G=8, K=A0, V=A1, mask=A2, slot=A3)
    d.update(kw)
    return rs.PagesDesc(*[d[x] for x in ("n_pages", "page", "vcap", "H", "dh", "G", "K", "V", "mask", "slot")])


@pytest.mark.parametrize("kw,status,word", [
    (dict(page=8), 2, "pages of 8"), (dict(page=48), 2, "pages of 48"), (dict(page=512), 2, "pages of 512"),
    (dict(dh=96), 2, "head dim"), (dict(G=33), 2, "G=33"), (dict(G=12), 1, "divide"), (dict(H=0), 1, "H >= 1"),
    (dict(n_pages=-1), 1, "n_pages"), (dict(vcap=-1), 1, "vcap"), (dict(K=None), 1, "non-NULL"),
    (dict(V=None), 1, "non-NULL"), (dict(mask=None), 1, "non-NULL"), (dict(slot=None), 1, "non-NULL"),
    (dict(K=ctypes.c_void_p(0x10000008)), 2, "16 bytes"), (dict(V=ctypes.c_void_p(0x10000008)), 2, "16"),
    (dict(H=1 << 20, page=256), 2, "2 GiB"),
])
def test_pages_validation(lib, kw, status, word):
    pg = _pages(**kw)
    calls = [
        lambda: lib.rolesub_cache_append(ctypes.byref(pg), rs.BF16, 1, 1, A0, 0, A0, 0, A0, A0, 2, A0, None, None),
        lambda: lib.rolesub_attend_paged(ctypes.byref(pg), rs.BF16, 1, max(pg.H, 1), 1, A0, 0, A0, 2, A0, None, 0, None, 0.0,
                                         A0, rs.BF16, None, 1.0, None, 0, A0, 1 << 40, None),
        lambda: lib.rolesub_cache_compact(ctypes.byref(pg), ctypes.byref(pg), rs.BF16, 1, A0, 2, A0, A0, 4, A0, 2, None, 0,
                                          None, 0, None),
    ]
    for call in calls:
        assert call() == status and word in _last()


def test_rotary_validation(lib):
    def call(B=1, T=2, H=4, Hkv=2, dh=64, dt=rs.BF16, q=A0, qs=0, k=A1, ks=0, pos=A2, na=3, f=A2, ax=A2, n=32, qo=A3,
             ko=ctypes.c_void_p(0x50000000)):
        return lib.rolesub_rotary(B, T, H, Hkv, dh, dt, q, qs, k, ks, pos, na, f, ax, n, 0, 0, qo, ko, None)
    assert call(dt=7) == 2 and call(dh=96) == 2 and call(B=-1) == 1 and call(na=0) == 2 and call(na=9) == 2
    assert call(n=0) == 1 and call(n=33) == 1
    assert call(H=0) == 1 and call(q=None, k=None) == 1 and call(pos=None) == 1 and call(qo=None) == 1
    assert call(qs=100) == 1 and "stride" in _last()
    assert call(qs=260) == 2 and "16 bytes" in _last()
    assert call(q=ctypes.c_void_p(0x10000004)) == 2
    assert call(qo=ctypes.c_void_p(0x10000010)) == 1 and "overlaps" in _last()
    assert call(qo=A1) == 1 and call(ko=A3) == 1
    assert call(q=A0, k=A0, qo=A0, ko=A0, H=2) == 1 and call(q=A0, k=A0, qo=A0, H=2) == 1  # one tensor turned twice
    # a query and a key of one fused row that share dims, in place
    near = ctypes.c_void_p(0x10000000 + 3 * 64 * 2)
    assert call(qs=512, ks=512, k=near, qo=A0, ko=near) == 1 and "overlaps" in _last()
    assert call(qs=512, ks=640, k=ctypes.c_void_p(0x10000000 + 4 * 64 * 2), qo=A0) == 1
    assert call(B=0, q=A0) == 0
    assert call(B=1 << 20, T=1 << 10) == 2 and "too many" in _last()


def test_append_validation(lib):
    def call(B=1, T=2, k=A0, ks=0, zs=0, mask=A0, table=A0, mp=2, lens=A0):
        return lib.rolesub_cache_append(ctypes.byref(_pages()), rs.BF16, B, T, k, ks, A0, zs, mask, table, mp, lens, None,
                                        None)
    assert call(B=-1) == 1 and call(mp=-1) == 1 and call(mask=None) == 1 and call(table=None) == 1 and call(lens=None) == 1
    assert call(k=None) == 1 and call(ks=127) == 1 and call(ks=132) == 2 and call(zs=12) == 1
    assert call(B=0) == 0 and call(T=0) == 0 and call(mp=0) == 0
    assert call(B=1 << 16, T=1 << 16) == 2
    assert lib.rolesub_cache_append(None, rs.BF16, 1, 1, A0, 0, A0, 0, A0, A0, 2, A0, None, None) == 1
    assert lib.rolesub_cache_append(ctypes.byref(_pages()), 9, 1, 1, A0, 0, A0, 0, A0, A0, 2, A0, None, None) == 2


def test_attend_paged_validation(lib):
    big = 1 << 40

    def call(B=1, Hq=4, Tq=1, q=A0, qs=0, table=A0, mp=2, lens=A0, ml=0, R=None, scale=0.0, out=A0, odt=rs.BF16, mi=None,
             decay=1.0, mo=None, ld=0, ws=A0, wsb=big, dt=rs.BF16):
        return lib.rolesub_attend_paged(ctypes.byref(_pages()), dt, B, Hq, Tq, q, qs, table, mp, lens, None, ml, R, scale, out,
                                        odt, mi, decay, mo, ld, ws, wsb, None)
    assert call(Hq=3) == 1 and "multiple" in _last()
    assert call(Hq=0) == 1 and call(odt=7) == 2 and call(dt=rs.F32, odt=rs.BF16) == 2
    assert call(scale=float("inf")) == 1 and call(decay=-1.0) == 1 and call(decay=float("nan")) == 1
    assert call(q=None) == 1 and call(lens=None) == 1 and call(table=None) == 1 and call(out=None) == 1
    assert call(ml=-1) == 1 and call(B=-1) == 1 and call(Tq=-1) == 1
    assert call(mi=A0) == 1 and "without mass_out" in _last()
    assert call(mo=A0, ld=31) == 1 and "mass_ld" in _last()
    assert call(mi=A0, mo=ctypes.c_void_p(0x10000010), ld=32) == 1 and "overlap" in _last()
    assert call(mp=100, ws=None) == 1 and "workspace" in _last()  # splits need one
    assert call(mp=100, wsb=16) == 1 and call(ws=ctypes.c_void_p(0x10000004)) == 1
    assert call(mo=A1, ld=32, wsb=16) == 1 and "workspace" in _last()  # and weights
    assert call(R=ctypes.c_void_p(0x10000008)) == 2 and call(out=ctypes.c_void_p(0x10000008)) == 2 and call(q=ctypes.c_void_p(0x10000008)) == 2
    assert call(qs=260) == 2 and call(qs=64) == 1
    assert call(mp=1 << 27) == 2 and "max_len" in _last()
    assert call(B=0) == 0 and call(Tq=0) == 0
    assert call(B=1 << 20, Tq=64) == 2


def test_attend_paged_workspace_grows(lib):
    def size(B, Tq, ml, mass=0, Hq=4):
        return lib.rolesub_attend_paged_workspace_size(ctypes.byref(_pages()), B, Hq, Tq, ml, mass)
    for mass in (0, 1):
        for a in (lambda x: size(x, 1, 3000, mass), lambda x: size(3, x, 3000, mass), lambda x: size(3, 1, 40 * x, mass),
                  lambda x: size(1, x, 131072, mass)):
            got = [a(x) for x in range(1, 400)]
            assert all(p <= q for p, q in zip(got, got[1:]))
    assert size(0, 1, 100) == 0 and size(1, 0, 100) == 0 and size(1, 1, 0) == 0


def test_evict_validation(lib):
    def call(B=1, ml=40, mass=A0, ld=40, lens=A0, keep=8, first=2, recent=2, idx=A0, n=A0, ws=A0, wsb=1 << 40):
        return lib.rolesub_evict_tokens(B, ml, mass, ld, lens, keep, first, recent, idx, n, ws, wsb, None)
    assert call(keep=0) == 1 and call(first=-1) == 1 and call(recent=7) == 1 and call(first=2 ** 31 - 1, recent=2 ** 31 - 1) == 1
    assert call(ld=39) == 1 and call(B=-1) == 1 and call(ml=-1) == 1
    assert call(mass=None) == 1 and call(lens=None) == 1 and call(idx=None) == 1 and call(n=None) == 1
    assert call(B=0) == 0 and call(B=1 << 23) == 2
    assert call(ml=(1 << 30) + 1, ld=1 << 31) == 2
    size = lib.rolesub_evict_workspace_size
    got = [size(3, n) for n in (1, 4096, 16384, 16385, 40000, 131071, 524288, 524289, 10 ** 6, 10 ** 9)]
    assert got == sorted(got) and got[3] > 0 and size(4, 40000) >= size(3, 40000) and size(0, 40000) == 0
    assert call(ml=40000, ld=40000, ws=None) == 1 and "workspace" in _last()
    assert call(ml=40000, ld=40000, ws=ctypes.c_void_p(0x10000004)) == 1


def test_compact_validation(lib):
    def call(src=None, dst=None, B=1, keep=4, idx=A0, n=A0, table=A0, dt=A0, mi=None, mo=None, ld=40, old=40):
        return lib.rolesub_cache_compact(ctypes.byref(src or _pages()), ctypes.byref(dst or _pages()), rs.BF16, B, table, 2, idx,
                                         n, keep, dt, 2, mi, ld, mo, old, None)
    assert call(dst=_pages(page=32)) == 1 and call(dst=_pages(H=4)) == 1 and call(dst=_pages(G=4)) == 1
    assert call(idx=None) == 1 and call(n=None) == 1 and call(table=None) == 1 and call(dt=None) == 1
    assert call(mi=A0) == 1 and "go together" in _last()
    assert call(mi=A0, mo=A1, old=3) == 1 and call(mi=A0, mo=A0) == 1 and call(mi=A0, mo=A1, ld=-1) == 1
    assert call(B=-1) == 1 and call(keep=-1) == 1 and call(B=0) == 0 and call(keep=0) == 0
    assert call(keep=1 << 30, B=64) == 2
