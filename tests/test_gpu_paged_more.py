"""Normed heads, appends from projections, drafted trees and few pages of long histories,
on the GPU against the float64 oracle of the paged cache.

Tolerances. u = 2^-24, half a step of 32 bits. Attention: as in test_gpu_paged.py. A norm: a
head's sum of dh squares is off by 16 u at most (eight or four squares a lane, five steps
between lanes, the squares themselves), its root by half of that, v_rsq_f32 by 2 u more and
the sum with eps by 1; weight times cosine, two products, their sum and the root's
factor by 6: with the turn's own 4e-7 (see _rotary_tol there) 2 max|n| (4e-7 + 18 u) in
all, and the output's rounding. Copies, choices and masks are exact."""
import numpy as np
import pytest
import torch

import paper_2608_18410_amd as rs
from oracle import paged as O
from paper_2608_18410_amd.pipeline import accept_layer, decode_layer, draft_layer, page_count
from tests._gpu_util import DEV
from tests.test_gpu_paged import EPS, HALF, bf, case, dev, f32, full_cache, i32, ints, num, rotations, to_np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    rs.load()


def same(a, b):
    """Equal bits."""
    bits = {2: torch.int16, 4: i32}[a.element_size()]
    return torch.equal(a.contiguous().view(bits), b.contiguous().view(bits))


def words(sets, T):
    return torch.from_numpy(O.tree_words(sets, T).view(np.int32)).to(DEV)


def random_parents(rng, B, T):
    return np.array([[j - 1 if rng.random() < 0.5 else rng.integers(-1, j) for j in range(T)] for _ in range(B)])


# ---- norm ------------------------------------------------------------------

def _norm_tol(n, y, dtype):
    a = np.abs(n).max(-1, keepdims=True)
    e = 2 * a * (4e-7 + 18 * 2.0 ** -24)
    return e + HALF[dtype] * (np.abs(y) + e)


def _turns(rng, B, T, A, pairs):
    pos = rng.integers(-100, 5000, (B, T, A))
    pos[0, 0] = 0
    f = (10000.0 ** (-np.arange(pairs) / pairs)).astype(np.float32)
    ax = rng.integers(0, A, pairs).astype(np.uint8)
    ax[0] = A if pairs > 1 else 0  # an axis that is none: not turned
    return pos, f, ax, torch.from_numpy(f).to(DEV), torch.from_numpy(ax).to(DEV)


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("dh,pairs", [(64, 32), (128, 64), (128, 32), (128, 24), (64, 13), (64, 1), (128, 63), (128, 3)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rotary(dtype, dh, pairs, interleaved):
    rng = np.random.default_rng(pairs + dh)
    for B, T in ((1, 1), (2, 5), (3, 700)):
        q, k = dev(rng.standard_normal((B, T, 6, dh)), dtype), dev(3 * rng.standard_normal((B, T, 3, dh)), dtype)
        wq, wk = dev(rng.standard_normal(dh), dtype), dev(rng.standard_normal(dh), dtype)
        pos, f, ax, ft, axt = _turns(rng, B, T, 3, pairs)
        got = rs.norm_rotary(q, k, wq, wk, 1e-5, ints(pos), ft, axt, interleaved=interleaved)
        few = slice(0, min(T, 5)), slice(max(0, T - 3), T)
        for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
            for sl in few:
                n = O.norm(num(x[:, sl]), num(w), np.float32(1e-5))
                ref = O.rotary(n, pos[:, sl], f, ax, interleaved)
                assert (np.abs(num(y[:, sl]) - ref) <= _norm_tol(n, ref, dtype)).all()
        # one tensor, and one that is not normed
        plain = rs.rotary(q, k, ints(pos), ft, axt, interleaved=interleaved)
        a, b = rs.norm_rotary(q, k, None, wk, 1e-5, ints(pos), ft, axt, interleaved=interleaved)
        assert same(a, plain[0]) and same(b, got[1])
        a, b = rs.norm_rotary(None, k, None, None, 1e-5, ints(pos), ft, axt, interleaved=interleaved)
        assert a is None and same(b, plain[1])


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("pairs", [64, 40, 61])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rotary_views_and_in_place(dtype, pairs, interleaved):
    rng = np.random.default_rng(5)
    B, T, H, Hkv, dh = 3, 7, 5, 2, 128
    qkv = dev(rng.standard_normal((B, T, (H + 2 * Hkv) * dh)), dtype)
    qkv[..., (H + Hkv) * dh:] = float("nan")
    q = qkv[..., :H * dh].unflatten(2, (H, dh))
    k = qkv[..., H * dh:(H + Hkv) * dh].unflatten(2, (Hkv, dh))
    w = dev(rng.standard_normal((2, dh)), dtype)
    pos, f = ints(rng.integers(0, 999, (B, T, 2))), torch.rand(pairs, device=DEV)
    ax = torch.randint(0, 2, (pairs,), device=DEV, dtype=torch.uint8)
    args = (w[0].contiguous(), w[1].contiguous(), 1e-6, pos, f, ax, interleaved)
    want = rs.norm_rotary(q.contiguous(), k.contiguous(), *args)
    got = rs.norm_rotary(q, k, *args)
    assert same(got[0], want[0]) and same(got[1], want[1]) and torch.isfinite(want[0]).all() and torch.isfinite(want[1]).all()
    keep = qkv[..., (H + Hkv) * dh:].clone()
    r = rs.norm_rotary(q, k, *args, out=(q, k))
    assert r[0] is q and same(q, want[0]) and same(k, want[1]) and same(qkv[..., (H + Hkv) * dh:], keep)
    with pytest.raises(rs.RolesubError, match="overlaps"):
        rs.norm_rotary(q, None, *args, out=(qkv.flatten()[8 * dh:8 * dh + B * T * H * dh].view(B, T, H, dh), None))
    empty = rs.norm_rotary(q[:0], k[:0], *args[:3], pos[:0], f, ax)
    assert empty[0].shape == (0, T, H, dh)


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rotary_extreme_heads(dtype, interleaved):
    rng = np.random.default_rng(6)
    dh, n = 128, 48
    x = rng.standard_normal((1, 8, 5, dh))
    x[0, 0] *= 1e30  # squares past 32 bits
    x[0, 1] *= 1e-30  # and below them: eps alone counts
    x[0, 2] = 0.0
    x[0, 3, 1, 5] = 3e38
    q = dev(x, dtype)
    w = dev(np.ones(dh), dtype)
    pos, f = rng.integers(0, 99, (1, 8, 1)), rng.random(n).astype(np.float32)
    run = lambda y: rs.norm_rotary(y, None, w, None, 1e-6, ints(pos), torch.from_numpy(f).to(DEV), interleaved=interleaved)[0]  # noqa: E731
    got = run(q)
    nn = O.norm(num(q), num(w), np.float32(1e-6))
    ref = O.rotary(nn, pos, f, None, interleaved)
    assert (np.abs(num(got) - ref) <= _norm_tol(nn, ref, dtype) + 1e-37).all()
    # an infinity: NaN in its place (and its pair's), zeros elsewhere in its head, nothing in others
    for bad in (float("inf"), float("nan")):
        q2 = q.clone()
        q2[0, 5, 2, 100] = bad  # past the pairs
        q2[0, 6, 3, 0] = bad
        y = run(q2)
        other = [(t, h) for t in range(8) for h in range(5) if (t, h) not in ((5, 2), (6, 3))]
        assert all(same(y[0, t, h], got[0, t, h]) for t, h in other)
        if bad != bad:
            assert torch.isnan(y[0, 5, 2]).all() and torch.isnan(y[0, 6, 3]).all()
            continue
        at = torch.isnan(y[0, 5, 2])
        assert at[100] and at.sum() == 1 and not y[0, 5, 2][~at].any()
        at = torch.isnan(y[0, 6, 3])
        assert at[0] and at[1 if interleaved else n] and at.sum() == 2 and not y[0, 6, 3][~at].any()


# ---- append ------------------------------------------------------------------

def _chain(c, q, k, v, mask, t, n, pos, f, ax, R, wq, wk, eps, il, n_new):
    """The separate calls."""
    if wk is None and wq is None:
        tq, tk = rs.rotary(q, k, pos, f, ax, interleaved=il)
    else:
        tq, tk = rs.norm_rotary(q, k, wq, wk, eps, pos, f, ax, interleaved=il)
    z = v.contiguous() if R is None else rs.rotate_values(v.contiguous(), R)
    rs.cache_append(c, tk, z, mask, t, n, n_new)
    return tq


def check_append(rng, lens, T, P=16, H=2, rep=2, dh=64, G=8, dtype=bf, R=True, norm=True, il=False, pairs=None, ragged=False,
                 fused=False, with_q=True, kmax=None, vcap=None, table=None, width=None):
    B = len(lens)
    width = width or page_count(max(max(lens), 0) + T, P)
    c = full_cache(rng, B * width + 2, P, H, dh, G, kmax or G, dtype, vcap)
    if table is None:
        table = ints(rng.permutation(B * width + 2)[: B * width].reshape(B, width))
    pairs = pairs or dh // 2
    if fused:
        qkv = dev(rng.standard_normal((B, T, (rep + 2) * H * dh)), dtype)
        q, k, v = (x.unflatten(2, (-1, dh)) for x in qkv.split((rep * H * dh, H * dh, H * dh), 2))
    else:
        q, k, v = (dev(rng.standard_normal((B, T, h, dh)), dtype) for h in (rep * H, H, H))
    q = q if with_q else None
    mask = ints(rng.integers(0, 1 << min(G, 30), (B, T)))
    pos, _, _, f, ax = _turns(rng, B, T, 3, pairs)
    w = [dev(rng.standard_normal(dh), dtype) if norm else None for _ in range(2)]
    Rm = rotations(rng, H, dh, dtype) if R else None
    n_new = ints(rng.integers(-1, T + 2, B)) if ragged else None
    d = rs.PagedCache(*(x.clone() for x in c.tensors()))
    n = ints(lens)
    want = _chain(d, q, k, v, mask, table, n, ints(pos), f, ax, Rm, w[0] if with_q else None, w[1], 1e-5, il, n_new)
    got = rs.append_rotary(c, k, v, mask, table, n, ints(pos), f, ax, R=Rm, q=q, q_weight=w[0] if with_q else None, k_weight=w[1],
                           eps=1e-5, interleaved=il, n_new=n_new)
    torch.cuda.synchronize()
    assert (got is None and want is None) or same(got, want)
    for name, a, b in zip(("K", "V", "mask", "slot"), c.tensors(), d.tensors()):
        assert same(a, b), (name, int((a != b).sum()))
    return c


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("dh,G", [(64, 8), (128, 8), (128, 1), (128, 32), (64, 32), (64, 16), (128, 2)])
@pytest.mark.parametrize("R", [True, False])
def test_append_rotary_gives_the_separate_calls_bits(dtype, dh, G, R):
    rng = np.random.default_rng(dh + G)
    for T in (1, 3, 40):
        check_append(rng, [0, 1, 15, 16, 37], T, dh=dh, G=G, dtype=dtype, R=R, ragged=T == 40, norm=T != 3)


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
def test_append_rotary_pages(dtype, P):
    rng = np.random.default_rng(P)
    check_append(rng, [0, 5, P - 1, P, 2 * P + 3], 300, P=P, H=3, rep=1, G=4, dtype=dtype, fused=True)
    check_append(rng, [0, 5, P - 1, P, 2 * P + 3], 300, P=P, H=1, rep=5, dh=128, dtype=dtype, ragged=True, with_q=False)


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("pairs", [32, 24, 31, 1])
@pytest.mark.parametrize("il", [False, True])
def test_append_rotary_pairs(dtype, pairs, il):
    rng = np.random.default_rng(pairs)
    check_append(rng, [3, 20], 70, dtype=dtype, pairs=pairs, il=il)
    check_append(rng, [3, 20], 2, dtype=dtype, pairs=pairs, il=il, norm=False, fused=True)


@pytest.mark.parametrize("dtype", [bf, f32])
def test_append_rotary_many_heads_and_tokens(dtype):
    rng = np.random.default_rng(1)
    check_append(rng, [0] * 3 + [100], 1100, P=64, H=4, rep=4, dh=128, dtype=dtype, fused=True)
    check_append(rng, list(range(40)), 1, H=9, rep=3, dh=128, dtype=dtype)


@pytest.mark.parametrize("dtype", [bf, f32])
def test_append_rotary_dropped_tokens(dtype):
    rng = np.random.default_rng(2)
    # the table ends among the new tokens; lengths outside it; pages that are none
    check_append(rng, [20, -3, 1000, 33], 30, dtype=dtype, width=3)
    t = ints([[1, -1, 3], [4, 5, 10 ** 6], [-7, -7, -7], [8, 9, 2]])
    check_append(rng, [20, 5, 3, 40], 30, dtype=dtype, table=t, width=3)
    check_append(rng, [20, 5, 3, 40], 30, dtype=dtype, table=t, width=3, R=False)
    # fewer slots than groups
    check_append(rng, [20, 5], 30, dtype=dtype, vcap=17)
    c = full_cache(rng, 3, 16, 2, 64, 8, 8, dtype)
    before = [x.clone() for x in c.tensors()]
    e = lambda *s, dt=dtype: torch.zeros(s, device=DEV, dtype=dt)  # noqa: E731
    # no page a sequence: the queries alone
    q = dev(rng.standard_normal((2, 3, 4, 64)), dtype)
    f = torch.rand(32, device=DEV)
    got = rs.append_rotary(c, e(2, 3, 2, 64), e(2, 3, 2, 64), e(2, 3, dt=i32), e(2, 0, dt=i32), e(2, dt=i32), ints([[1, 2, 3]] * 2), f, q=q)
    assert same(got, rs.rotary(q, None, ints([[1, 2, 3]] * 2), f)[0])
    rs.append_rotary(c, e(0, 3, 2, 64), e(0, 3, 2, 64), e(0, 3, dt=i32), e(0, 1, dt=i32), e(0, dt=i32), e(0, 3, dt=i32), f)
    assert all(same(a, b) for a, b in zip(before, c.tensors()))


def test_append_rotary_queries_in_place():
    rng = np.random.default_rng(3)
    c = full_cache(rng, 4, 16, 2, 64, 8, 8, bf)
    d = rs.PagedCache(*(x.clone() for x in c.tensors()))
    qkv = dev(rng.standard_normal((2, 5, 8 * 64)), bf)
    q, k, v = (x.unflatten(2, (-1, 64)) for x in qkv.split((256, 128, 128), 2))
    args = (ints(rng.integers(0, 256, (2, 5))), ints([[0, 1], [2, 3]]), ints([3, 14]), ints(rng.integers(0, 9, (2, 5))),
            torch.rand(32, device=DEV))
    want = rs.append_rotary(c, k, v, *args, q=q)
    kv = qkv[..., 256:].clone()
    assert rs.append_rotary(d, k, v, *args, q=q, q_out=q) is q
    assert same(q, want) and same(qkv[..., 256:], kv) and all(same(a, b) for a, b in zip(c.tensors(), d.tensors()))
    with pytest.raises(rs.RolesubError, match="overlaps"):
        rs.append_rotary(d, k, v, *args, q=q, q_out=d.K.flatten()[:2 * 5 * 256].view(2, 5, 4, 64))


# ---- drafted trees -----------------------------------------------------------

@pytest.mark.parametrize("T", [1, 2, 8, 31, 32, 33, 64, 65, 100, 255, 256])
def test_tree_masks(T):
    rng = np.random.default_rng(T)
    par = random_parents(rng, 5, T)
    par[1] = np.arange(T) - 1  # a chain
    par[2] = -1  # all children of the cached tokens
    par[3] = rng.integers(-9, 400, T)  # numbers that are no earlier token's
    par[4] = np.where(rng.random(T) < 0.3, np.array([2 ** 31 - 1, -2 ** 31, T, T - 1])[rng.integers(0, 4, T)], par[4])
    tree, depth = rs.tree_masks(ints(par))
    sets, deep = O.tree_masks(par)
    assert np.array_equal(tree.cpu().numpy().view(np.uint32), O.tree_words(sets, T)) and depth.tolist() == deep
    t2, d2 = rs.tree_masks(ints(par), out=(torch.empty_like(tree), None))
    assert torch.equal(t2, tree) and d2 is None


def check_tree(q, c, t, n, sets, R=None, n_new=None, scale=0.0, max_len=0, out_dtype=None, workspace=None, sees=None):
    cn = to_np(c)
    nn = None if n_new is None else n_new.cpu().numpy()
    sees = O.tree_sees(cn, t.cpu().numpy(), n.cpu().numpy(), sets, q.shape[1], nn, max_len)
    ref, size, A = O.attend_over(num(q), cn, sees, None if R is None else num(R), scale)
    out = rs.attend_tree(q, c, t, n, words(sets, q.shape[1]), R, n_new=n_new, scale=scale, max_len=max_len, out_dtype=out_dtype,
                         workspace=workspace)
    torch.cuda.synchronize()
    return _held(out, ref, size, A, q.shape[3], t.shape[1] * c.K.shape[2])


def _held(out, ref, size, A, dh, n):
    rel = 2 * EPS * (dh + 8) * A + 2.0 ** -17 + EPS * (n + 2 * dh + 40)
    err, tol = np.abs(num(out) - ref), rel * size + HALF[out.dtype] * (np.abs(ref) + rel * size)
    assert (err <= tol).all(), (float(err.max()), float((err / np.maximum(tol, 1e-300)).max()))
    return out


def _trees(rng, B, T):
    return O.tree_masks(random_parents(rng, B, T))[0]


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("dh,G", [(64, 8), (128, 8), (128, 1), (128, 32), (64, 32), (64, 16)])
def test_tree_lengths(dtype, dh, G):
    T = 7
    base = [0, 1, 9, 15, 16, 17, 25, 31, 32, 57, 64, 120, 121, 128, 129, 250]
    rng, c, t, n, q = case(1, [x + T for x in base], dh=dh, G=G, dtype=dtype, Tq=T)
    check_tree(q, c, t, n - T, _trees(rng, len(base), T), rotations(rng, 2, dh, dtype))


@pytest.mark.parametrize("H,rep,Tq", [(1, 1, 1), (2, 4, 3), (5, 1, 16), (1, 2, 17), (2, 1, 33), (1, 4, 24), (1, 1, 64), (3, 1, 65),
                                      (1, 3, 70), (1, 1, 256)])
@pytest.mark.parametrize("dtype,dh", [(bf, 64), (bf, 128), (f32, 64)])
def test_tree_rows(H, rep, Tq, dtype, dh):
    base = [37, 0, 161]
    rng, c, t, n, q = case(3, [x + Tq for x in base], H=H, rep=rep, Tq=Tq, dh=dh, dtype=dtype)
    sets = _trees(rng, 3, Tq)
    R = rotations(rng, H, dh, dtype)
    few = ints([Tq, Tq // 2, -1])
    check_tree(q, c, t, ints(base), sets, R, out_dtype=f32)
    out = check_tree(q, c, t, ints(base), sets, R, n_new=few)
    assert not out[2].any() and not out[1, Tq // 2:].any()
    check_tree(q, c, t, ints(base), sets[:1], n_new=ints([Tq + 5, 1, 0]))  # one tree for all
    # any bits: not a tree's
    anyb = [[set(np.flatnonzero(rng.random(Tq) < 0.5).tolist()) for _ in range(Tq)] for _ in range(3)]
    check_tree(q, c, t, ints(base), anyb, n_new=few)


@pytest.mark.parametrize("dtype,dh", [(bf, 128), (f32, 64)])
@pytest.mark.parametrize("Tq", [3, 40])
def test_tree_rows_that_see_nothing(dtype, dh, Tq):
    rng, c, t, n, q = case(5, [Tq + 9, Tq], H=2, rep=2, Tq=Tq, dh=dh, dtype=dtype)
    sets, R = _trees(rng, 2, Tq), rotations(rng, 2, dh, dtype)
    for x in (c.K, c.V):
        x.fill_(float("nan"))
    for kw in (dict(n_new=ints([0, -3])), dict(table=t[:, :0].contiguous()), dict(table=torch.full_like(t, -1)),
               dict(tree=torch.zeros(2, Tq, (Tq + 31) // 32, dtype=torch.int32, device=q.device), lens=ints([0, 0]))):
        out = torch.full_like(q, 7.0)
        rs.attend_tree(q, c, kw.get("table", t), kw.get("lens", ints([9, 0])), kw.get("tree", words(sets, Tq)), R,
                       n_new=kw.get("n_new"), out=out)
        assert not out.any(), kw
    # and over the queries themselves
    inplace = q.clone()
    for x in (c.K, c.V):
        x.copy_(torch.randn(x.shape, device=q.device).to(dtype))
    args = c, t, ints([9, 0]), words(sets, Tq), R
    assert same(rs.attend_tree(inplace, *args, out=inplace), rs.attend_tree(q, *args))


# as many row tiles as the card holds: whole sequences in one split, the longest first
@pytest.mark.parametrize("B,H,rep,Tq,top", [(61, 9, 1, 17, 700), (64, 8, 4, 5, 90), (300, 2, 1, 24, 520), (64, 8, 1, 33, 5000)])
@pytest.mark.parametrize("dtype,dh", [(bf, 64), (bf, 128), (f32, 64), (f32, 128)])
def test_tree_whole_sequences(B, H, rep, Tq, top, dtype, dh):
    base = [0, 1, 33, top] + [(29 * i) % 83 for i in range(B - 4)]
    rng, c, t, n, q = case(4, [x + Tq for x in base], P=32, H=H, rep=rep, Tq=Tq, dh=dh, dtype=dtype)
    few = ints([Tq if i % 5 else i % (Tq + 1) for i in range(B)])
    check_tree(q, c, t, ints(base), _trees(rng, B, Tq), rotations(rng, H, dh, dtype), n_new=few)


@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [bf, f32])
def test_tree_pages_and_bounds(P, dtype):
    T = 20
    base = [1, P - 1, P, P + 1, 2 * P + 5, 200]
    rng, c, t, n, q = case(2, [x + T for x in base], P=P, H=3, G=4, Tq=T, dtype=dtype)
    sets = _trees(rng, len(base), T)
    check_tree(q, c, t, ints(base), sets)
    check_tree(q, c, t, ints(base), sets, max_len=P + 9, scale=-0.2)  # ends among the cached or the drafted tokens
    t2 = t.clone()
    t2[1, 0], t2[3, :] = -1, 10 ** 6
    out = check_tree(q, c, t2, ints([-4, P - 1, P, P + 1, 10 ** 6, t.shape[1] * P - 3]), sets)
    assert not out[3].any()


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("rep,T", [(1, 3), (2, 12), (1, 40)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_tree_what_is_not_seen_does_not_reach(dtype, rep, T, bad):
    base = [30, 61]
    rng, c, t, n, q = case(8, [x + T for x in base], rep=rep, Tq=T, kmin=1, dtype=dtype)
    par = np.array([[-1, 0, 0] + [1] * (T - 3)] * 2)
    sets = O.tree_masks(par)[0]
    clean = check_tree(q, c, t, ints(base), sets)
    tok = base[0] + 2  # the third drafted token: no one's ancestor
    pg, r = int(t[0, tok // 16]), tok % 16
    s, k = int(c.slot[pg, r]), bin(int(c.mask[pg, r]) & 255).count("1")
    c.V[pg, :, s:s + k] = bad
    if (base[1] + T) % 16:  # rows behind the last sequence's tokens
        c.K[int(t[1, (base[1] + T) // 16]), :, (base[1] + T) % 16:] = bad
    out = rs.attend_tree(q, c, t, ints(base), words(sets, T))
    ok = torch.isfinite(out[0]).all(-1).all(-1)
    assert ok.tolist() == [j != 2 for j in range(T)]
    tol = 4 * HALF[dtype] * np.abs(num(clean)) + 1e-4
    assert (np.abs(num(out[0]) - num(clean[0]))[num(ok) > 0] <= tol[0][num(ok) > 0]).all()
    assert (np.abs(num(out[1]) - num(clean[1])) <= tol[1]).all()


@pytest.mark.parametrize("dtype,n", [(bf, 9000), (f32, 5000)])
@pytest.mark.parametrize("T", [4, 30])
def test_tree_of_a_chain_is_causal_attention(dtype, n, T):
    """Long histories in many splits: rows that see lens + j + 1 tokens."""
    rng, c, t, _, q = case(13, [n + T, n // 3 + T, T], P=64, H=2, rep=2, dh=128, Tq=T, dtype=dtype)
    base = ints([n, n // 3, 0])
    sets = O.tree_masks(np.array([np.arange(T) - 1]))[0]
    got = rs.attend_tree(q, c, t, base, words(sets, T), max_len=n + T, out_dtype=f32)
    vis = base[:, None] + torch.arange(1, T + 1, device=DEV, dtype=i32)
    want = rs.attend_paged(q, c, t, base + T, visible=vis, max_len=n + T, out_dtype=f32)
    assert bool(((got - want).abs() <= 2 ** -20 * want.abs() + 1e-6).all())


def _state(c):
    return {x: y.copy() for x, y in to_np(c).items()}


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("P,T", [(16, 1), (16, 5), (16, 60), (32, 33), (64, 256), (256, 100)])
@pytest.mark.parametrize("dh,G", [(64, 8), (128, 32), (64, 32), (128, 1)])
def test_accept(dtype, P, T, dh, G):
    rng = np.random.default_rng(T)
    lens = [0, 1, 15, 16, 37, 100, P - 1, 5]
    B, H = len(lens), 5
    width = page_count(max(lens) + T, P)
    c = full_cache(rng, B * width, P, H, dh, G, G, dtype)
    t = ints(rng.permutation(B * width).reshape(B, width))
    k, z = dev(rng.standard_normal((2, B, T, H, dh)), dtype)
    mask = ints(rng.integers(0, 1 << min(G, 30), (B, T)))
    rs.cache_append(c, k, z, mask, t, ints(lens))
    for shared in (False, True):
        sets = _trees(rng, 1 if shared else B, T)
        if not shared:
            sets[0] = [set(range(T)) for _ in range(T)]  # everything stays
            sets[1] = [set(np.flatnonzero(rng.random(T) < 0.7).tolist()) for _ in range(T)]
        leaf = ints(list(rng.integers(0, T, B - 3)) + [-1, T, T - 1])
        d = rs.PagedCache(*(x.clone() for x in c.tensors()))
        cn = _state(d)
        want = O.accept(cn, t.cpu().numpy(), lens, sets, leaf.tolist())
        got = rs.cache_accept(d, t, ints(lens), words(sets, T), leaf)
        assert got.tolist() == want.tolist()
        for x, y in _state(d).items():
            assert np.array_equal(y, cn[x]), x
        # the next tokens go on from there
        k2, z2 = dev(rng.standard_normal((2, B, 2, H, dh)), dtype)
        m2 = ints(rng.integers(0, 1 << min(G, 30), (B, 2)))
        t3 = torch.cat((t, torch.full((B, 1), -1, device=DEV, dtype=i32)), 1)
        rs.cache_append(d, k2, z2, m2, t3, got)
        O.append(cn, num(k2), num(z2), m2.cpu().numpy().view(np.uint32), t3.cpu().numpy(), want)
        for x, y in _state(d).items():
            assert np.array_equal(y, cn[x]), x


@pytest.mark.parametrize("dtype", [bf, f32])
def test_accept_pages_that_are_none_and_short_tables(dtype):
    rng = np.random.default_rng(4)
    c = full_cache(rng, 9, 16, 3, 64, 8, 8, dtype)
    t = ints([[0, -1, 2], [3, 4, 5], [6, 7, 8]])
    lens, T = [10, 30, -3], 25  # the second's drafted tokens pass its table
    k, z = dev(rng.standard_normal((2, 3, T, 3, 64)), dtype)
    rs.cache_append(c, k, z, ints(rng.integers(0, 256, (3, T))), t, ints(lens))
    sets = [[{1, 2, 9, 20, 24}] * T, [{0, 3, 17, 22}] * T, [{4, 5}] * T]
    cn = _state(c)
    want = O.accept(cn, t.cpu().numpy(), lens, sets, [0, 1, 2])
    got = rs.cache_accept(c, t, ints(lens), words(sets, T), ints([0, 1, 2]))
    assert got.tolist() == want.tolist()
    for x, y in _state(c).items():
        assert np.array_equal(y, cn[x]), x
    before = [x.clone() for x in c.tensors()]
    n = rs.cache_accept(c, t, ints([1, 2, 3]), torch.zeros((3, 0, 0), device=DEV, dtype=i32), ints([0, 0, 0]))
    assert n.tolist() == [1, 2, 3] and all(same(a, b) for a, b in zip(before, c.tensors()))


# ---- few pages ---------------------------------------------------------------

@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("P,dh", [(16, 64), (64, 128), (256, 128), (32, 64)])
def test_page_bounds(dtype, P, dh):
    rng = np.random.default_rng(P)
    lens = [0, 1, P - 1, P, P + 1, 3 * P, 200, 5000, -2]
    c = full_cache(rng, 40, P, 3, dh, 8, 8, dtype)
    c.K[3, :, 2] = float("nan")
    c.K[4, 0, :, 5] = float("nan")
    c.K[5, 1, 1, 1], c.K[5, 1, 0, 2] = float("inf"), float("-inf")
    t = ints(rng.permutation(36).reshape(9, 4))
    t[5, 1] = -1
    t[6, 0] = 10 ** 6
    for T in (1, 2, P, P + 1, 10 ** 6, 0):
        b = dev(rng.standard_normal((40, 3, 2, dh)), dtype)
        ref = num(b).copy()
        O.page_bounds(to_np(c), t.cpu().numpy(), lens, ref, T)
        assert rs.page_bounds(c, t, ints(lens), b, T) is b
        assert np.array_equal(num(b), ref), T


def bounds_of(c):
    b = torch.stack((c.K.amin(2), c.K.amax(2)), 2)
    return b.contiguous()


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("H,rep,Tq,dh", [(1, 1, 1, 64), (2, 4, 1, 128), (3, 1, 3, 64), (1, 5, 2, 128), (2, 2, 9, 64)])
def test_select_pages(dtype, H, rep, Tq, dh):
    P = 16
    lens = [0, 1, 16, 17, 500, 1100, 1300, 3000]
    rng, c, t, n, q = case(5, lens, P=P, H=H, rep=rep, Tq=Tq, dh=dh, dtype=dtype)
    bd = bounds_of(c)
    bd[t[4, 5].long()] = bd[t[4, 9].long()]  # equal scores
    bd[t[4, 7].long()] = float("nan")
    t[5, 3] = -1
    cn, tn = to_np(c), t.cpu().numpy()
    vis = ints(rng.integers(-5, 3000, (len(lens), Tq)))
    for n_sel, first, recent, v, ml in ((1, 0, 0, None, 0), (7, 1, 2, None, 0), (7, 0, 7, vis, 0), (40, 3, 5, vis, 0), (200, 1, 1, None, 0),
                                        (9, 0, 1, None, 700)):
        want = O.select_pages(num(q), cn, num(bd), tn, lens, n_sel, first, recent, None if v is None else v.cpu().numpy(), ml)
        got = rs.select_pages(q, c, bd, t, n, n_sel, first, recent, visible=v, max_len=ml)
        assert np.array_equal(got.cpu().numpy(), want), (n_sel, first, recent)


def test_select_pages_infinite_bounds():
    rng, c, t, n, q = case(6, [900, 640], P=16, H=2, rep=2, dh=128)
    bd = bounds_of(c)
    for i in range(0, 50, 3):
        bd[int(t[0, i]), i % 2, i % 4 // 2, i] = float("inf") if i % 4 // 2 else float("-inf")
    bd[int(t[1, 4]), :, 0], bd[int(t[1, 4]), :, 1] = float("inf"), float("-inf")  # a page of NaN
    q[1, 0, 1, 3] = 0.0
    want = O.select_pages(num(q), to_np(c), num(bd), t.cpu().numpy(), [900, 640], 6)
    assert np.array_equal(rs.select_pages(q, c, bd, t, n, 6).cpu().numpy(), want)


@pytest.mark.parametrize("dtype", [bf, f32])
def test_select_pages_of_long_histories(dtype):
    """More pages than one workgroup holds, against a sort on the GPU."""
    P, W, H, dh = 16, 20000, 1, 64
    g = torch.Generator(device=DEV).manual_seed(1)
    N = W + 1
    c = rs.PagedCache(torch.zeros((N, H, P, dh), device=DEV, dtype=dtype), torch.zeros((N, H, 16, 8), device=DEV, dtype=dtype),
                      torch.zeros((N, P), device=DEV, dtype=i32), torch.zeros((N, P), device=DEV, dtype=i32))
    bd = torch.randn((N, H, 2, dh), generator=g, device=DEV, dtype=dtype)
    t = torch.randperm(N, generator=g, device=DEV)[None, :W].int().contiguous()
    q = torch.randn((1, 2, 3, dh), generator=g, device=DEV, dtype=dtype)
    got = rs.select_pages(q, c, bd, t, ints([W * P - 3]), 333, 2, 4)
    x = q.double()[0]
    b = bd.double()[t[0].long(), 0]
    score = torch.where(x[:, :, None] < 0, x[:, :, None] * b[:, 0], x[:, :, None] * b[:, 1]).sum(-1).float().amax(1)  # [2, W]
    score[:, :2] = score[:, -4:] = float("inf")
    want = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :333].sort(1).values
    assert torch.equal(got[0, :, 0].long(), want)


def check_selected(q, c, t, n, sel, R=None, scale=0.0, visible=None, out_dtype=None, workspace=None):
    cn = to_np(c)
    sees = O.selected_sees(cn, t.cpu().numpy(), n.cpu().numpy(), sel.cpu().numpy(), None if visible is None else visible.cpu().numpy())
    ref, size, A = O.attend_over(num(q), cn, sees, None if R is None else num(R), scale)
    out = rs.attend_selected(q, c, t, n, sel, R, scale=scale, visible=visible, out_dtype=out_dtype, workspace=workspace)
    torch.cuda.synchronize()
    return _held(out, ref, size, A, q.shape[3], sel.shape[3] * c.K.shape[2])


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("dh,G", [(64, 8), (128, 8), (128, 1), (128, 32), (64, 32), (64, 16)])
def test_selected_lists(dtype, dh, G):
    """Any order, a page twice, numbers that are none, a page that ends a sequence in the middle."""
    lens = [0, 1, 15, 16, 17, 100, 161, 300]
    rng, c, t, n, q = case(1, lens, dh=dh, G=G, dtype=dtype, rep=2)
    for n_sel in (1, 2, 7, 21):
        sel = ints(rng.integers(-2, t.shape[1] + 2, (len(lens), 1, 2, n_sel)))
        sel[7, 0, 0, 0], sel[5, 0, 1, 0] = 18, 6
        check_selected(q, c, t, n, sel, rotations(rng, 2, dh, dtype), out_dtype=f32)
    sel[:] = ints([2 ** 31 - 1, -2 ** 31, 10 ** 6, -1] * 5 + [0])
    check_selected(q, c, t, n, sel)
    assert not rs.attend_selected(q, c, t, n, sel * 0 - 1).any()


@pytest.mark.parametrize("H,rep,Tq", [(1, 1, 1), (2, 4, 3), (3, 17, 2), (1, 33, 3), (1, 40, 1), (2, 1, 9)])
@pytest.mark.parametrize("dtype,dh", [(bf, 64), (bf, 128), (f32, 64), (f32, 128)])
def test_selected_rows(H, rep, Tq, dtype, dh):
    lens = [37, 0, 161]
    rng, c, t, n, q = case(3, lens, H=H, rep=rep, Tq=Tq, dh=dh, dtype=dtype)
    sel = ints(rng.integers(-1, t.shape[1], (3, Tq, H, 9)))
    vis = ints(rng.integers(-2, 200, (3, Tq)))
    check_selected(q, c, t, n, sel, rotations(rng, H, dh, dtype), visible=vis)
    check_selected(q, c, t, n, sel, scale=-0.3)


@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [bf, f32])
def test_selected_pages(P, dtype):
    rng, c, t, n, q = case(2, [1, P - 1, P, P + 1, 2 * P + 5, 300], P=P, H=3, G=4, dtype=dtype)
    sel = ints(rng.integers(0, t.shape[1], (6, 1, 3, 3)))
    check_selected(q, c, t, n, sel)
    t[1, 0], t[4, 1], t[5, 0] = -1, 10 ** 6, c.K.shape[0]
    check_selected(q, c, t, ints([P * t.shape[1] + 9, 10 ** 6, -1, P, 2 * P + 5, 2 ** 31 - 1]), sel)


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("rep", [1, 40])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_selected_what_is_not_listed_does_not_reach(dtype, rep, bad):
    rng, c, t, n, q = case(8, [70, 130], H=1, rep=rep, Tq=2, kmin=1, dtype=dtype)
    sel = ints([[[[0, 4]], [[1, 3]]], [[[8, 0]], [[2, 8]]]])
    vis = ints([[70, 60], [130, 129]])
    clean = check_selected(q, c, t, n, sel, visible=vis)
    for b, tok in ((0, 70), (1, 130)):  # dead rows of the last page
        pg = int(t[b, tok // 16])
        c.K[pg, :, tok % 16:] = bad
        c.V[pg, :, int(c.slot[pg, tok % 16]):] = bad
    c.K[int(t[0, 2])] = bad
    c.V[int(t[1, 1])] = bad
    assert torch.equal(clean, rs.attend_selected(q, c, t, n, sel, visible=vis))
    pg, r = int(t[1, 8]), 1  # token 129: seen by the first query only
    s, k = int(c.slot[pg, r]), bin(int(c.mask[pg, r]) & 255).count("1")
    c.V[pg, :, s:s + k] = bad
    out = rs.attend_selected(q, c, t, n, sel, visible=vis)
    assert torch.equal(torch.isfinite(out[1]).all(-1).all(-1), torch.tensor([False, True], device=DEV))
    assert torch.equal(out[0], clean[0])
    assert (np.abs(num(out[1, 1]) - num(clean[1, 1])) <= 4 * HALF[dtype] * np.abs(num(clean[1, 1])) + 1e-4).all()


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("rep", [1, 4])
def test_selected_all_pages_is_attend_paged(dtype, rep):
    """Many pages in many splits, lists that end early."""
    lens = [9000, 4321, 64, 0]
    rng, c, t, n, q = case(13, lens, P=64, H=2, rep=rep, dh=128, dtype=dtype)
    W = t.shape[1]
    sel = torch.full((4, 1, 2, W), -1, device=DEV, dtype=i32)
    for b, x in enumerate(lens):
        m = page_count(x, 64)
        sel[b, 0, :, :m] = ints([rng.permutation(m) for _ in range(2)]) if m else sel[b, 0, :, :0]
    got = rs.attend_selected(q, c, t, n, sel, out_dtype=f32)
    want = rs.attend_paged(q, c, t, n, out_dtype=f32)
    assert bool(((got - want).abs() <= 2 ** -20 * want.abs() + 1e-6).all())
    assert torch.equal(got, rs.attend_selected(q, c, t, n, sel, out_dtype=f32))


def test_workspaces_of_larger_calls_serve_smaller_ones():
    rng, c, t, n, q = case(11, [300, 161, 5], rep=4, Tq=5, dtype=bf)
    bd, sets = bounds_of(c), _trees(rng, 3, 5)
    need = max(rs.attend_tree_workspace_size(c, 3, 8, 5, 304), rs.select_pages_workspace_size(c, 3, 5, 304),
               rs.attend_selected_workspace_size(c, 3, 8, 5, 9))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    for b, tq, ml, k in ((3, 5, 304, 9), (1, 5, 304, 9), (3, 1, 304, 3), (2, 3, 17, 1), (1, 1, 129, 2)):
        a = (q[:b, :tq].contiguous(), c)
        at = (t[:b].contiguous(), n[:b].contiguous())
        w = words([[s & set(range(tq)) for s in row[:tq]] for row in sets[:b]], tq)
        ws.fill_(255)
        assert torch.equal(rs.attend_tree(*a, at[0], at[1] - tq, w, max_len=ml, workspace=ws), rs.attend_tree(*a, at[0], at[1] - tq, w, max_len=ml))
        ws.fill_(255)
        sel = rs.select_pages(*a, bd, *at, k, max_len=ml, workspace=ws)
        assert torch.equal(sel, rs.select_pages(*a, bd, *at, k, max_len=ml))
        ws.fill_(255)
        assert torch.equal(rs.attend_selected(*a, *at, sel, workspace=ws), rs.attend_selected(*a, *at, sel))


# ---- together ----------------------------------------------------------------

class Model:
    """One layer's weights and a generator of its inputs."""

    def __init__(self, seed, dtype, B, H=2, rep=2, dh=64, G=8, P=16, W=12):
        self.rng = np.random.default_rng(seed)
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.dtype, self.B, self.H, self.rep, self.dh, self.G = dtype, B, H, rep, dh, G
        self.R = rotations(self.rng, H, dh, dtype)
        self.w = [dev(1 + 0.1 * self.rng.standard_normal(dh), dtype) for _ in range(2)]
        self.f = torch.from_numpy((100.0 ** (-np.arange(dh // 2) / (dh // 2))).astype(np.float32)).to(DEV)
        self.budget = rs.make_budget(rs.TOPK, (3, 5, G, 1))
        self.cache = full_cache(self.rng, B * W, P, H, dh, G, G, dtype)
        self.table = ints(self.rng.permutation(B * W).reshape(B, W))

    def tokens(self, T):
        r = lambda *s, dtype=self.dtype: torch.randn(s, generator=self.g, device=DEV, dtype=dtype)  # noqa: E731
        return dict(q=r(self.B, T, self.H * self.rep, self.dh), k=r(self.B, T, self.H, self.dh), v=r(self.B, T, self.H, self.dh),
                    types=torch.randint(0, 4, (self.B, T), generator=self.g, device=DEV).to(torch.uint8),
                    scores=r(self.B, T, self.G, dtype=f32))

    def clone(self):
        return rs.PagedCache(*(x.clone() for x in self.cache.tensors()))

    def common(self, x, cache):
        return (None, x["q"], x["k"], x["v"], x["types"], self.R, self.budget, self.G, cache, self.table)

    def kw(self):
        return dict(inv_freq=self.f, q_weight=self.w[0], k_weight=self.w[1])


def _pick(x, b_path):
    """Of each sequence b its tokens b_path[b] ([B] lists of one length)."""
    at = torch.tensor(b_path, device=DEV)
    return {n: torch.stack([t[b, at[b]] for b in range(t.shape[0])]).contiguous() for n, t in x.items()}


def _apart(m):
    """How far two calls that sum the same terms may be apart before they round: weights of 17 bits and 2^-17 of the rest
    (see _held), of sums no larger than sqrt(dh) (a rotation's rows) times the largest value."""
    return 2.0 ** -15 * m.dh ** 0.5 * float(m.cache.V.abs().max())


@pytest.mark.parametrize("dtype", [bf, f32])
def test_drafted_tokens_decode_as_if_one_by_one(dtype):
    """Two rounds of draft, attend and accept, against a cache that is decoded along each path."""
    m = Model(1, dtype, 3)
    prompt = m.tokens(40)
    zero, lens = ints([0] * 3), ints([40] * 3)
    pos = torch.arange(40, device=DEV, dtype=i32).expand(3, 40).contiguous()
    decode_layer(*m.common(prompt, m.cache), zero, lens, positions=pos, scores_in=prompt["scores"], visible=pos + 1, **m.kw())
    plain = m.clone()
    T, par = 9, [[-1, 0, 0, 1, 2, 2, -1, 6, 4], [-1, 0, 1, 2, 3, 4, 5, 6, 7], [-1, -1, -1, 0, 1, 2, 3, 4, 6]]
    for step in range(2):
        x = m.tokens(T)
        tree, depth = rs.tree_masks(ints(par))
        out = draft_layer(*m.common(x, m.cache), lens, tree, positions=lens[:, None] + depth, scores_in=x["scores"], **m.kw())
        sets = O.tree_masks(par)[0]
        leaf = [5, 2, 6] if step == 0 else [8, 3, 8]
        paths = [sorted(sets[b][leaf[b]]) for b in range(3)]
        assert len({len(p) for p in paths}) == 1
        n1 = lens
        for i in range(len(paths[0])):
            y = _pick(x, [[p[i]] for p in paths])
            one = decode_layer(*m.common(y, plain), n1, n1 + 1, positions=n1[:, None], scores_in=y["scores"], **m.kw())
            want, got = num(one), np.stack([num(out[b, paths[b][i]]) for b in range(3)])[:, None]
            assert (np.abs(want - got) <= 2 * HALF[dtype] * np.abs(want) + _apart(m)).all()
            n1 = n1 + 1
        lens = accept_layer(m.cache, m.table, lens, tree, ints(leaf))
        assert torch.equal(lens, n1)
        a, b = to_np(m.cache), to_np(plain)
        for s in range(3):
            for t in range(int(lens[s])):
                u, v = O.token(a, m.table[s].tolist(), t), O.token(b, m.table[s].tolist(), t)
                assert all(np.array_equal(p, q) for p, q in zip(u, v)), (s, t)
    y = m.tokens(1)
    outs = [decode_layer(*m.common(y, c), lens, lens + 1, positions=lens[:, None], scores_in=y["scores"], **m.kw()) for c in (m.cache, plain)]
    assert torch.equal(*outs)


@pytest.mark.parametrize("dtype", [bf, f32])
def test_decoding_over_few_pages(dtype):
    m = Model(2, dtype, 3)
    bounds = torch.zeros((m.cache.K.shape[0], m.H, 2, m.dh), device=DEV, dtype=dtype)
    lens = ints([0] * 3)
    plain = m.clone()
    for T in (70, 1, 1, 9, 16, 1, 33):
        x = m.tokens(T)
        pos = lens[:, None] + torch.arange(T, device=DEV, dtype=i32)
        kw = dict(positions=pos, scores_in=x["scores"], visible=pos + 1, **m.kw())
        few = decode_layer(*m.common(x, m.cache), lens, lens + T, bounds=bounds, n_sel=4, **kw)
        everything = decode_layer(*m.common(x, plain), lens, lens + T, **kw)
        lens = lens + T
        assert all(same(a, b) for a, b in zip(m.cache.tensors(), plain.tensors()))
        ref = num(bounds).copy()
        O.page_bounds(to_np(m.cache), m.table.cpu().numpy(), lens.tolist(), ref, 10 ** 6)
        assert np.array_equal(num(bounds), ref)
        # (the turned queries as the layer makes them)
        q = rs.norm_rotary(x["q"], None, m.w[0], None, 1e-6, pos, m.f)[0]
        sel = rs.select_pages(q, m.cache, bounds, m.table, lens, 4, 1, 2, visible=pos + 1)
        assert torch.equal(few, rs.attend_selected(q, m.cache, m.table, lens, sel, m.R, visible=pos + 1))
        seen = ((pos + 1).max() + 15) // 16
        if int(seen) <= 4:
            err = (few.double() - everything.double()).abs()
            assert bool((err <= 2 * HALF[dtype] * everything.double().abs() + _apart(m)).all())
        whole = rs.select_pages(q, m.cache, bounds, m.table, lens, m.table.shape[1], visible=pos + 1)
        got = rs.attend_selected(q, m.cache, m.table, lens, whole, m.R, visible=pos + 1)
        err = (got.double() - everything.double()).abs()
        assert bool((err <= 2 * HALF[dtype] * everything.double().abs() + _apart(m)).all())


def _buffers(m, T):
    return dict(tree=torch.empty((m.B, T, 1), device=DEV, dtype=i32), depth=torch.empty((m.B, T), device=DEV, dtype=i32),
                out=torch.empty((m.B, T, m.H * m.rep, m.dh), device=DEV, dtype=m.dtype), new=torch.empty(m.B, device=DEV, dtype=i32),
                one=torch.empty((m.B, 1, m.H * m.rep, m.dh), device=DEV, dtype=m.dtype),
                ws=torch.empty(max(rs.attend_tree_workspace_size(m.cache, m.B, m.H * m.rep, T, 192),
                                   rs.attend_selected_workspace_size(m.cache, m.B, m.H * m.rep, 1, 5), 1), device=DEV, dtype=torch.uint8))


def test_draft_accept_and_few_pages_graph_replays():
    """A whole step captured: masks, drafted tokens, the accepted path, then a token over few pages."""
    m = Model(3, bf, 3)
    T, start = 6, ints([30, 15, 61])
    other, orig = m.clone(), m.clone()
    x, y = m.tokens(T), m.tokens(1)
    par, leaf, lens = ints([[-1, 0, 0, 1, 2, 4]] * 3), ints([5, 3, 0]), start.clone()
    bounds = torch.stack((m.cache.K.amin(2), m.cache.K.amax(2)), 2).contiguous()
    first_bounds, b = bounds.clone(), _buffers(m, T)

    def step(cache, bounds, x, y, lens, b):
        rs.tree_masks(par, out=(b["tree"], b["depth"]))
        draft_layer(*m.common(x, cache), lens, b["tree"], positions=lens[:, None] + b["depth"], scores_in=x["scores"], workspace=b["ws"],
                    out=b["out"], **m.kw())
        accept_layer(cache, m.table, lens, b["tree"], leaf, bounds=bounds, new_lens=b["new"])
        decode_layer(*m.common(y, cache), b["new"], b["new"] + 1, positions=b["new"][:, None], scores_in=y["scores"], bounds=bounds,
                     n_sel=5, workspace=b["ws"], out=b["one"], **m.kw())
        lens.copy_(b["new"] + 1)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(m.cache, bounds, x, y, lens, b)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(m.cache, bounds, x, y, lens, b)
    lens.copy_(start)
    bounds.copy_(first_bounds)
    for a, o in zip(m.cache.tensors(), orig.tensors()):
        a.copy_(o)
    lens1, bounds1, b1 = start.clone(), first_bounds.clone(), _buffers(m, T)
    for i in range(6):
        for d, n in ((x, m.tokens(T)), (y, m.tokens(1))):
            for k in d:
                d[k].copy_(n[k])
        par.copy_(ints(random_parents(m.rng, 3, T)))
        leaf.copy_(ints(m.rng.integers(-1, T, 3)))
        for k in ("tree", "depth", "new"):
            b[k].fill_(-7)
        b["out"].fill_(float("nan"))
        b["ws"].fill_(255)
        graph.replay()
        step(other, bounds1, x, y, lens1, b1)
        torch.cuda.synchronize()
        assert torch.equal(lens, lens1) and same(bounds, bounds1), i
        for k in ("tree", "depth", "out", "new", "one"):
            assert same(b[k], b1[k]), (i, k)
        for a, o in zip(m.cache.tensors(), other.tensors()):
            assert same(a, o), i


@pytest.mark.parametrize("B,H,top", [(3, 2, 900), (64, 8, 600)])  # split, whole
def test_trees_of_many_rows_graph_replays(B, H, top):
    Tq = 33
    rng, c, t, n, q = case(6, [top + Tq] * 2 + [(37 * i) % 71 + Tq for i in range(B - 2)], P=32, H=H, Tq=Tq, dh=128, dtype=bf)
    sets, R, lens, few = words(_trees(rng, B, Tq), Tq), rotations(rng, H, 128, bf), n - Tq, ints([Tq] * B)
    max_len = t.shape[1] * 32
    ws = [torch.empty(max(rs.attend_tree_workspace_size(c, B, H, Tq, max_len), 1), device=DEV, dtype=torch.uint8) for _ in range(2)]
    out = [torch.empty_like(q) for _ in range(2)]

    def step(i):
        rs.attend_tree(q, c, t, lens, sets, R, n_new=few, workspace=ws[i], out=out[i])

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(0)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for i in range(5):
        q.copy_(torch.randn(q.shape, device=DEV).to(bf))
        lens.copy_(ints(np.roll(lens.cpu().numpy(), 1)))  # other sequences are the long ones; tables that end give what is there
        few.copy_(ints(rng.integers(0, Tq + 1, B)))
        out[0].fill_(float("nan"))
        ws[0].fill_(255)
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        assert same(*out), i


def test_two_streams_at_once():
    """Two layers with their own caches and workspaces give the bits of one after the other; what a call with stream= makes
    is ready for the caller after the stream."""
    ms = [Model(i, bf, 3, dh=128, W=40) for i in (4, 5)]
    xs = [m.tokens(9) for m in ms]
    lens = ints([500, 300, 7])
    par = ints([[-1, 0, 1, 1, 2, 3, 4, 5, 6]] * 3)
    caches = [[m.clone() for m in ms] for _ in range(2)]

    def run(i, c, stream=None):
        m, x = ms[i], xs[i]
        tree, depth = rs.tree_masks(par)
        out = draft_layer(*m.common(x, c), lens, tree, positions=lens[:, None] + depth, scores_in=x["scores"], stream=stream, **m.kw())
        new = accept_layer(c, m.table, lens, tree, ints([8, 4, -1]), stream=stream)
        return out, new

    want = [run(i, caches[0][i]) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        cs = [m.clone() for m in ms]
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        got = [run(i, cs[i], streams[i]) for i in range(2)]
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        for i in range(2):
            assert same(got[i][0], want[i][0]) and torch.equal(got[i][1], want[i][1])
            assert all(same(a, b) for a, b in zip(cs[i].tensors(), caches[0][i].tensors()))


def test_far_pages():
    """Pages, bounds and queries whose bytes lie past 2^32 of their tensors."""
    H, P, dh, G, N = 8, 256, 128, 8, 4300
    K = torch.empty((N, H, P, dh), dtype=bf, device=DEV)
    V = torch.empty((N, H, P * G, dh // G), dtype=bf, device=DEV)
    rng = np.random.default_rng(12)
    small = full_cache(rng, 4, P, H, dh, G, G, bf)
    c = rs.PagedCache(K, V, torch.zeros((N, P), dtype=i32, device=DEV), torch.zeros((N, P), dtype=i32, device=DEV))
    far = [N - 1, N - 2, 4100, 0]
    for i, p in enumerate(far):
        for a, b in zip(c.tensors(), small.tensors()):
            a[p] = b[i]
    t, ts = ints([[N - 1, 4100], [N - 2, 0]]), ints([[0, 2], [1, 3]])
    T = 5
    k, v, q = (dev(rng.standard_normal((2, T, h, dh)), bf) for h in (H, H, H))
    mask, pos, f = ints(rng.integers(0, 256, (2, T))), ints(rng.integers(0, 99, (2, T))), torch.rand(64, device=DEV)
    n = ints([300, 255])
    R = rotations(rng, H, dh, bf)
    bd, bs = torch.zeros((N, H, 2, dh), device=DEV, dtype=bf), torch.zeros((4, H, 2, dh), device=DEV, dtype=bf)
    tree, _ = rs.tree_masks(ints([[-1, 0, 0, 2, 1]] * 2))
    outs = []
    for cache, table, b in ((c, t, bd), (small, ts, bs)):
        o = [rs.append_rotary(cache, k, v, mask, table, n, pos, f, R=R, q=q)]
        o.append(rs.attend_tree(q, cache, table, n, tree, R))
        o.append(rs.cache_accept(cache, table, n, tree, ints([3, 4])))
        rs.page_bounds(cache, table, o[-1], b, 10 ** 6)
        o.append(rs.select_pages(q, cache, b, table, o[2], 1))
        o.append(rs.attend_selected(q, cache, table, o[2], o[3], R))
        outs.append(o)
    for a, b in zip(*outs):
        assert same(a, b)
    for i, p in enumerate(far):
        assert same(bd[p], bs[i])
        for a, b in zip(c.tensors(), small.tensors()):
            assert same(a[p], b[i])
