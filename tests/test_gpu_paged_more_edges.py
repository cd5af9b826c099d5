"""What the paged cache's normed heads, appends, drafted trees and chosen pages do at the edges of
their ranges, on the GPU against the float64 oracle. Tolerances as in test_gpu_paged_more.py."""
import numpy as np
import pytest
import torch

import paper_2608_18410_amd as rs
from oracle import paged as O
from paper_2608_18410_amd.pipeline import decode_layer, page_count
from tests._gpu_util import DEV
from tests.test_gpu_paged import bf, case, dev, f32, full_cache, i32, ints, num, rotations, to_np
from tests.test_gpu_paged_more import Model, _norm_tol, _trees, check_append, same, words

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    rs.load()


# ---- the type of the outputs -------------------------------------------------

@pytest.mark.parametrize("rep,Tq,top", [(1, 8, 305), (4, 3, 900), (3, 20, 700), (1, 100, 200)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("R", [False, True])
def test_tree_outputs_round_the_same_sums(rep, Tq, top, dh, R):
    """bfloat16 outputs are the float32 ones rounded: the same weights and sums come before."""
    rng, c, t, n, q = case(21, [top + Tq, top // 3 + Tq, Tq], H=2, rep=rep, Tq=Tq, dh=dh, dtype=bf)
    args = q, c, t, n - Tq, words(_trees(rng, 3, Tq), Tq), rotations(rng, 2, dh, bf) if R else None
    one = rs.attend_tree(*args)
    assert same(one, rs.attend_tree(*args, out_dtype=f32).to(bf))
    for _ in range(3):
        assert same(one, rs.attend_tree(*args))


@pytest.mark.parametrize("rep,n_sel", [(1, 24), (4, 40), (20, 9), (40, 33)])
@pytest.mark.parametrize("dh", [64, 128])
def test_selected_outputs_round_the_same_sums(rep, n_sel, dh):
    rng, c, t, n, q = case(22, [700, 161, 1], H=2, rep=rep, Tq=2, dh=dh, dtype=bf)
    sel = ints(rng.integers(-1, t.shape[1], (3, 2, 2, n_sel)))
    args = q, c, t, n, sel, rotations(rng, 2, dh, bf)
    one = rs.attend_selected(*args)
    assert same(one, rs.attend_selected(*args, out_dtype=f32).to(bf))
    for _ in range(3):
        assert same(one, rs.attend_selected(*args))


# ---- norms at the ends of the range --------------------------------------------

def _ends(rng, dh):
    """Heads, weights and eps at the ends of float32's range."""
    x = rng.standard_normal((9, dh))
    sign = np.where(rng.random((9, dh)) < 0.5, -1.0, 1.0)
    big = np.minimum(np.abs(x) * 1e38, 3.3e38) * sign
    two = 1e-3 * x
    two[:, 7], two[:, dh - 1] = 3e38, -3e38
    one, w = np.ones(dh), rng.standard_normal(dh)
    return [
        ("every dim near the largest number", 3.3e38 * sign, one, 1e-6),
        ("squares whose sum passes 2^256", 4e37 * sign, w, 1e-6),
        ("a few of them", two, one, 1e-6),
        ("with weights", big, 8 * w, 1e-6),
        ("times the weight past the range", 1e15 * x, 1e30 * w, 1e-6),
        ("times the weight below the range", 1e-20 * x, 1e-30 * w, 1e-30),
        ("squares below the range and so is eps", 1e-22 * x, w, 1e-43),
        ("eps below the normal numbers", 1e-3 * x, w, 1e-40),
        ("zeros with eps below the normal numbers", 0 * x, w, 1e-44),
        ("eps near the largest number", 1e19 * x, 1e10 * w, 3e38),
    ]


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("dh,pairs", [(128, 64), (64, 16), (128, 61), (64, 3)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rotary_at_the_ends_of_the_range(dtype, dh, pairs, interleaved):
    rng = np.random.default_rng(31)
    pos, f = rng.integers(0, 99, (1, 3, 1)), rng.random(pairs).astype(np.float32)
    ft = torch.from_numpy(f).to(DEV)
    for name, x, w, eps in _ends(rng, dh):
        q, wt = dev(x.reshape(1, 3, 3, dh), dtype), dev(w, dtype)
        assert torch.isfinite(q).all() and torch.isfinite(wt).all()
        n = O.norm(num(q), num(wt), np.float32(eps))
        ref = O.rotary(n, pos, f, None, interleaved)
        got, _ = rs.norm_rotary(q, None, wt, None, float(np.float32(eps)), ints(pos), ft, interleaved=interleaved)
        assert torch.isfinite(got).all(), name
        # (below 2^-126 a float32 number is off by 2^-150, a bfloat16 one by 2^-134)
        err = np.abs(num(got) - ref)
        assert (err <= _norm_tol(n, ref, dtype) + (2.0 ** -134 if dtype == bf else 2.0 ** -149)).all(), (name, float(err.max()))


def test_appended_keys_at_the_ends_of_the_range():
    rng = np.random.default_rng(32)
    for dtype in (bf, f32):
        for name, x, w, eps in _ends(rng, 64):
            c = full_cache(rng, 2, 16, 3, 64, 8, 8, dtype)
            k, wk, pos, f = dev(x.reshape(1, 3, 3, 64), dtype), dev(w, dtype), ints([[3, 1, 4]]), torch.rand(32, device=DEV)
            rs.append_rotary(c, k, torch.zeros_like(k), ints([[1, 2, 3]]), ints([[1]]), ints([5]), pos, f, k_weight=wk, eps=float(np.float32(eps)))
            want = rs.norm_rotary(None, k, None, wk, float(np.float32(eps)), pos, f)[1]
            assert same(c.K[1, :, 5:8].transpose(0, 1), want[0]), name


# ---- bits that are only moved ---------------------------------------------------

def _payloads(rng, x):
    """x with NaN of every kind (quiet, signalling, negative, of any payload) in a tenth of its places."""
    bits = x.view({2: torch.int16, 4: i32}[x.element_size()])
    wide, top, low = (16, 0x7F80, 7) if x.element_size() == 2 else (32, 0x7F800000, 23)
    nan = top | rng.integers(1, 1 << low, tuple(x.shape)) | (rng.integers(0, 2, tuple(x.shape)) << (wide - 1))
    nan = np.where(nan >= 1 << (wide - 1), nan - (1 << wide), nan)
    put = torch.from_numpy(rng.random(tuple(x.shape)) < 0.1).to(DEV)
    bits.copy_(torch.where(put, torch.from_numpy(nan).to(DEV), bits.long()).to(bits.dtype))
    return x


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("pairs", [64, 32, 16, 61, 3])
@pytest.mark.parametrize("interleaved", [False, True])
def test_dims_that_are_not_turned_keep_their_bits(dtype, pairs, interleaved):
    rng = np.random.default_rng(41)
    q, k = (_payloads(rng, dev(rng.standard_normal((2, 9, h, 128)), dtype)) for h in (5, 2))
    pos, f = ints(rng.integers(0, 99, (2, 9, 2))), torch.rand(pairs, device=DEV)
    ax = torch.randint(0, 3, (pairs,), device=DEV, dtype=torch.uint8)  # a third of the pairs has no axis
    want = rs.rotary(q, k, pos, f, ax, interleaved=interleaved)
    got = rs.norm_rotary(q, k, None, None, 1e-6, pos, f, ax, interleaved=interleaved)
    e = torch.arange(128, device=DEV)
    j = (e // 2 if interleaved else torch.where(e < pairs, e, e - pairs)).clamp(max=pairs - 1)
    still = (e >= 2 * pairs) | (ax[j] >= 2)
    for x, y, z in ((q, *(o[0] for o in (got, want))), (k, *(o[1] for o in (got, want)))):
        assert same(y[..., still], x[..., still]) and same(z[..., still], x[..., still])
        # what a turn makes of a NaN is a NaN whose sign and payload IEEE 754 (6.2, 6.3) leaves open
        assert torch.equal(torch.isnan(y), torch.isnan(z)) and same(y.nan_to_num(1.0), z.nan_to_num(1.0))


@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("G", [8, 32])
def test_values_kept_as_they_are_keep_their_bits(dtype, G):
    rng = np.random.default_rng(42)
    for dh in (64, 128):
        c = full_cache(rng, 6, 16, 2, dh, G, G, dtype)
        d = rs.PagedCache(*(x.clone() for x in c.tensors()))
        k = dev(rng.standard_normal((2, 20, 2, dh)), dtype)
        v = _payloads(rng, dev(rng.standard_normal((2, 20, 2, dh)), dtype))
        mask, t, n = ints(rng.integers(0, 1 << min(G, 30), (2, 20))), ints([[0, 1, 2], [3, 4, 5]]), ints([5, 16])
        pos, f = ints(rng.integers(0, 99, (2, 20))), torch.rand(dh // 2, device=DEV)
        rs.append_rotary(c, k, v, mask, t, n, pos, f)
        rs.cache_append(d, rs.rotary(None, k, pos, f)[1], v, mask, t, n)
        assert all(same(a, b) for a, b in zip(c.tensors(), d.tensors()))


# ---- appends of many tokens and heads -------------------------------------------

@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("dh,P,R", [(128, 16, True), (64, 256, True), (128, 256, False), (64, 16, True), (128, 64, True)])
def test_append_rotary_long_runs(dtype, dh, P, R):
    """From 1025 groups of 64 tokens and a head on a workgroup takes 128 tokens."""
    rng = np.random.default_rng(51)
    check_append(rng, [0, 5, 300], 700, P=P, H=32, rep=1, dh=dh, dtype=dtype, R=R, ragged=True, fused=P == 256)
    check_append(rng, [9] * 7 + [250], 301, P=P, H=32, rep=1, dh=dh, G=32 if dh == 128 else 4, dtype=dtype, R=R, with_q=False)


# ---- choices among few and many pages ---------------------------------------------

def select_ref(q, bd, table, n_pages, P, lens, n_sel, first, recent, visible, max_len):
    """The oracle's choice, a sequence's pages at once."""
    B, Tq, Hq, dh = q.shape
    H = bd.shape[1]
    cap = table.shape[1] * P
    cap = min(cap, max_len) if max_len else cap
    sel = np.full((B, Tq, H, n_sel), -1, dtype=np.int32)
    for b in range(B):
        m0 = page_count(min(max(int(lens[b]), 0), cap), P)
        if m0 == 0:
            continue
        pg = table[b, :m0].long()
        there = (pg >= 0) & (pg < n_pages)
        lo, hi = bd[pg.clamp(0, n_pages - 1)].double().permute(2, 1, 0, 3)[:, :, None]  # [H, 1, m, dh]
        x = q[b].double().unflatten(1, (H, -1))
        for j in range(Tq):
            y = x[j][:, :, None]  # [H, rep, 1, dh]
            s = torch.where(y < 0, y * lo, y * hi).sum(-1).float()
            s = torch.where(torch.isnan(s).any(1) | ~there, torch.tensor(float("nan"), device=DEV), s.amax(1)).cpu().numpy()
            n = min(max(int(lens[b]), 0), cap)
            n = n if visible is None else min(n, max(int(visible[b, j]), 0))
            m = page_count(n, P)
            for g in range(H):
                mine = list(range(m))
                if m > n_sel:
                    free = np.arange(first, m - recent)
                    z = s[g, free]
                    order = np.lexsort((free, np.where(np.isnan(z), 0.0, -z), np.isnan(z)))
                    keep = free[order][: n_sel - first - recent].tolist()
                    mine = sorted(list(range(first)) + keep + list(range(m - recent, m)))
                sel[b, j, g, : len(mine)] = mine
    return sel


@pytest.mark.parametrize("W", [255, 511, 512, 513, 2000])
@pytest.mark.parametrize("dtype,dh", [(bf, 64), (bf, 128), (f32, 64), (f32, 128)])
@pytest.mark.parametrize("rep,Tq", [(1, 1), (4, 2), (5, 1)])
def test_select_pages_at_the_border_of_one_launch(W, dtype, dh, rep, Tq):
    P, H = 16, 2
    rng, g = np.random.default_rng(W + rep), torch.Generator(device=DEV).manual_seed(W)
    lens = [0, 1, W * P, 17, W * P - 5, 700, W * P + 99, -4]
    B, N = len(lens), W + 3
    c = rs.PagedCache(torch.zeros((N, H, P, dh), device=DEV, dtype=dtype), torch.zeros((N, H, 16, 8), device=DEV, dtype=dtype),
                      torch.zeros((N, P), device=DEV, dtype=i32), torch.zeros((N, P), device=DEV, dtype=i32))
    bd = torch.randn((N, H, 2, dh), generator=g, device=DEV, dtype=dtype)
    t = torch.stack([torch.randperm(N, generator=g, device=DEV)[:W] for _ in range(B)]).int()
    bd[t[2, 5].long()] = bd[t[2, 9].long()]  # equal scores
    bd[t[4, 50:90].long()] = bd[t[4, 9].long()].clone()
    bd[t[2, 7].long()] = float("nan")
    bd[t[4, 11].long(), 1, 0, 3] = float("-inf")
    t[4, 3], t[2, 20], t[6, 40] = -1, 10 ** 6, N
    q = torch.randn((B, Tq, rep * H, dh), generator=g, device=DEV, dtype=dtype)
    vis = ints(rng.integers(-5, W * P + 50, (B, Tq)))
    ws = torch.full((rs.select_pages_workspace_size(c, B, Tq, W * P),), 255, dtype=torch.uint8, device=DEV)
    for n_sel, first, recent, v, ml in ((1, 0, 0, None, 0), (7, 1, 2, None, 0), (9, 0, 9, vis, 0), (40, 3, 5, vis, 0), (W + 5, 1, 1, None, 0),
                                        (W - 1, 0, 0, None, 0), (9, 0, 1, None, W * P // 2 + 3)):
        want = select_ref(q, bd, t, N, P, lens, n_sel, first, recent, v, ml)
        got = rs.select_pages(q, c, bd, t, ints(lens), n_sel, first, recent, visible=v, max_len=ml, workspace=ws)
        assert np.array_equal(got.cpu().numpy(), want), (n_sel, first, recent)


# ---- bounds of shared pages ---------------------------------------------------

@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("B,H", [(2, 2), (7, 1), (70, 3), (200, 2), (300, 5), (260, 1)])
def test_bounds_of_a_shared_page_hold_for_all_its_sequences(dtype, B, H):
    """Sequences with the same first pages and lengths that end in one of them: its bounds are over
    the tokens of the longest, whichever comes last, and also where only its end is among the last T."""
    rng = np.random.default_rng(B)
    P, dh, W = 64, 128, 4
    c = full_cache(rng, 40 + B, P, H, dh, 8, 8, dtype)
    c.K[:, :, 1::2] *= 3  # later tokens widen the bounds
    table = rng.permutation(40)[:W][None].repeat(B, 0)
    table[1::3, 3] = 40 + np.arange(B)[1::3]  # a last page of its own
    for lens in ([P + 1 + (37 * i) % (2 * P) for i in range(B)], [P + 60 - i % 50 for i in range(B)], [3 * P + 1] + [P + 5] * (B - 1),
                 [P + 5] * (B - 1) + [3 * P + 1], [P] + [P + 9] * (B - 1)):
        for T in (1, 5, 10 ** 6):
            b = dev(rng.standard_normal((40 + B, H, 2, dh)), dtype)
            ref = num(b).copy()
            held = {}
            for s in range(B):
                for i in range(page_count(lens[s], P)):
                    held[table[s, i]] = max(held.get(table[s, i], 0), min(P, lens[s] - i * P))
            for s in range(B):
                for i in range(max(lens[s] - T, 0) // P, page_count(lens[s], P)):
                    k = num(c.K[int(table[s, i]), :, : held[table[s, i]]])
                    ref[table[s, i], :, 0], ref[table[s, i], :, 1] = k.min(1), k.max(1)
            for _ in range(3):
                again = b.clone()
                rs.page_bounds(c, ints(table), ints(lens), again, T)
                assert np.array_equal(num(again), ref), (lens[:4], T)


# ---- layers -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [bf, f32])
@pytest.mark.parametrize("T", [1, 4])
def test_few_pages_see_nothing_past_max_len(dtype, T):
    """A bound inside the last chosen page hides what attention over all pages hides too."""
    m = Model(61, dtype, 3)
    bounds = torch.zeros((m.cache.K.shape[0], m.H, 2, m.dh), device=DEV, dtype=dtype)
    lens = ints([60, 75, 70])
    rs.page_bounds(m.cache, m.table, lens, bounds, 10 ** 6)
    few, everything = m.clone(), m.clone()
    x = m.tokens(T)
    x["v"][:] = float("nan")  # the new tokens of the last two lie past the bound
    pos = lens[:, None] + torch.arange(T, device=DEV, dtype=i32)
    args = dict(positions=pos, scores_in=x["scores"], max_len=70, **m.kw())
    got = decode_layer(*m.common(x, few), lens, lens + T, n_sel=12, bounds=bounds, **args)
    want = decode_layer(*m.common(x, everything), lens, lens + T, **args)
    assert torch.isnan(want[0]).any() and not torch.isnan(want[1:]).any()
    assert not torch.isnan(got[1:]).any()
    half = 2.0 ** -8 if dtype == bf else 2.0 ** -24
    apart = 2.0 ** -15 * m.dh ** 0.5 * float(few.V[~torch.isnan(few.V)].abs().max())  # see _apart there
    assert bool(((got[1:].float() - want[1:].float()).abs() <= 2 * half * want[1:].float().abs() + apart).all())


@pytest.mark.parametrize("dtype", [bf, f32])
def test_layers_take_operands_that_lie_in_the_cache(dtype):
    """Queries, keys and values that are views of the pages: read before anything is appended."""
    m = Model(62, dtype, 2, rep=1)
    x = m.tokens(3)
    lens, pos = ints([20, 33]), ints([[20, 21, 22], [33, 34, 35]])
    n = 2 * 3 * m.H * m.dh
    for weights in (True, False):
        kw = dict(positions=pos, scores_in=x["scores"], **(m.kw() if weights else dict(inv_freq=m.f)))
        for i, name in enumerate(("q", "k", "v")):
            a, b = m.clone(), m.clone()
            src = (a.K if i < 2 else a.V).flatten()[i * n: (i + 1) * n].view(2, 3, m.H, m.dh)
            got = decode_layer(*m.common({**x, name: src}, a), lens, lens + 3, **kw)
            src = (b.K if i < 2 else b.V).flatten()[i * n: (i + 1) * n].view(2, 3, m.H, m.dh).clone()
            want = decode_layer(*m.common({**x, name: src}, b), lens, lens + 3, **kw)
            assert same(got, want) and all(same(u, v) for u, v in zip(a.tensors(), b.tensors())), name


@pytest.mark.parametrize("dtype", [bf, f32])
def test_a_layer_over_few_pages_shares_one_workspace(dtype):
    m = Model(63, dtype, 3)
    bounds = torch.zeros((m.cache.K.shape[0], m.H, 2, m.dh), device=DEV, dtype=dtype)
    lens = ints([60, 75, 170])
    rs.page_bounds(m.cache, m.table, lens, bounds, 10 ** 6)
    x = m.tokens(2)
    pos = lens[:, None] + torch.arange(2, device=DEV, dtype=i32)
    whole = m.table.shape[1] * 16
    small = rs.attend_selected_workspace_size(m.cache, 3, m.H * m.rep, 2, 5)
    both = max(small, rs.select_pages_workspace_size(m.cache, 3, 2, whole))
    outs = []
    for ws in (None, small, both):
        ws = None if ws is None else torch.full((max(ws, 1),), 255, dtype=torch.uint8, device=DEV)
        outs.append(decode_layer(*m.common(x, m.clone()), lens, lens + 2, positions=pos, scores_in=x["scores"], n_sel=5, bounds=bounds.clone(),
                                 workspace=ws, **m.kw()))
    assert same(outs[0], outs[1]) and same(outs[0], outs[2])
