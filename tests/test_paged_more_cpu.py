"""Normed heads, appends from projections, drafted trees and few pages of long histories
without a GPU: the oracle against textbook forms, the binding's shape checks, and the
library's refusals (all before anything is launched)."""
import ctypes
import re
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2608_18410_amd as rs
from oracle import paged as O
from paper_2608_18410_amd import build
from tests.test_mfma_waits import early_reads, functions
from tests.test_paged_cpu import _np_cache
from tests.test_stream_memory import allocations

bf, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


# ---- oracle ----------------------------------------------------------------

def test_oracle_norm():
    rng = np.random.default_rng(0)
    x, w = rng.standard_normal((2, 3, 4, 16)), rng.standard_normal(16)
    n = O.norm(x, w, 1e-6)
    np.testing.assert_allclose((n / w) ** 2 @ np.ones(16), 16 / (1 + 1e-6 / (x * x).mean(-1)), rtol=1e-12)
    np.testing.assert_allclose(O.norm(-3 * x, w, 9e-6), -n, rtol=1e-12)
    pos, f = rng.integers(0, 50, (2, 3, 1)), np.ones(8)
    y = O.norm_rotary(x, w, 1e-6, pos, f)
    z = (n[..., :8] + 1j * n[..., 8:]) * np.exp(1j * pos[..., None])
    np.testing.assert_allclose(y, np.concatenate((z.real, z.imag), -1), atol=1e-12)
    assert np.array_equal(O.norm_rotary(x, None, 1.0, pos, f), O.rotary(x, pos, f))


def test_oracle_tree():
    sets, depth = O.tree_masks([[-1, 0, 0, 2, 9, 4]])
    assert sets[0] == [{0}, {0, 1}, {0, 2}, {0, 2, 3}, {4}, {4, 5}] and depth == [[0, 1, 1, 2, 0, 1]]
    w = O.tree_words([[{0, 31, 32}] * 33], 33)
    assert w.shape == (1, 33, 2) and w[0, 5].tolist() == [2 ** 31 + 1, 1]


def test_oracle_tree_attention_is_that_of_each_path():
    """A row's output is the attention over its own continuation alone, appended to the cache."""
    rng = np.random.default_rng(1)
    H, rep, dh, G, P, n, T = 2, 2, 16, 4, 16, 21, 9
    par = [-1, 0, 0, 1, 2, 2, -1, 6, 4]
    sets = O.tree_masks([par])[0]
    k, z = rng.standard_normal((2, 1, n + T, H, dh))
    m = rng.integers(0, 16, (1, n + T))
    table, q = np.array([[3, 1]]), rng.standard_normal((1, T, H * rep, dh))
    c = _np_cache(4, H, P, dh, G, P * G)
    O.append(c, k, z, m, table, [0])
    out = O.attend_over(q, c, O.tree_sees(c, table, [n], sets, T))[0]
    for j in range(T):
        path = list(range(n)) + [n + i for i in sorted(sets[0][j])]
        d = _np_cache(4, H, P, dh, G, P * G)
        O.append(d, k[:, path], z[:, path], m[:, path], table, [0])
        np.testing.assert_allclose(out[:, j], O.attend(q[:, j:j + 1], d, table, [len(path)])[0][:, 0], atol=1e-12)
        # and what is kept of the cache, if this token is the last accepted one
        e = {x: c[x].copy() for x in c}
        assert O.accept(e, table, [n], sets, [j]).tolist() == [len(path)]
        for t in range(len(path)):
            a, b = O.token(e, table[0], t), O.token(d, table[0], t)
            assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_oracle_selection_bounds_every_key():
    rng = np.random.default_rng(2)
    H, rep, dh, P, W = 2, 3, 8, 16, 12
    c = dict(K=rng.standard_normal((W, H, P, dh)), V=np.zeros((W, H, P, 4)), mask=np.zeros((W, P)), slot=np.zeros((W, P)))
    table, q = rng.permutation(W)[None], rng.standard_normal((1, 1, H * rep, dh))
    b = np.zeros((W, H, 2, dh))
    O.page_bounds(c, table, [W * P], b, 10 ** 6)
    top = O.select_pages(q, c, b, table, [W * P], 1)
    for h in range(H):
        score = np.einsum("xd,wpd->wxp", q[0, 0, h * rep:(h + 1) * rep], c["K"][table[0], h]).max((1, 2))
        bound = [max((np.where(x < 0, x * b[p, h, 0], x * b[p, h, 1])).sum() for x in q[0, 0, h * rep:(h + 1) * rep]) for p in table[0]]
        assert (score <= np.array(bound) + 1e-12).all() and top[0, 0, h, 0] == int(np.argmax(bound))
    assert O.select_pages(q, c, b, table, [50], 6)[0, 0, 0].tolist() == [0, 1, 2, 3, -1, -1]
    sel = O.select_pages(q, c, b, table, [W * P], 5, first=1, recent=2)
    assert (sel[..., 0] == 0).all() and (sel[..., -2:] == [10, 11]).all()
    # listing every page is attention over all of them
    everything = np.tile(np.arange(W), (1, 1, H, 1))
    c["mask"][:] = 3
    c["slot"][:] = np.arange(P) * 2
    c["V"] = rng.standard_normal((W, H, P * 2, 4))
    got = O.attend_over(q, c, O.selected_sees(c, table, [W * P - 3], everything))[0]
    np.testing.assert_allclose(got, O.attend(q, c, table, [W * P - 3])[0], atol=1e-12)


# ---- binding ---------------------------------------------------------------

B, T, H, Hq, dh, G, P, N, W = 2, 3, 2, 4, 64, 8, 16, 5, 2


def z(*shape, dtype=bf):
    return torch.zeros(shape, dtype=dtype)


def cache():
    return rs.PagedCache(K=z(N, H, P, dh), V=z(N, H, P * 4, dh // G), mask=z(N, P, dtype=i32), slot=z(N, P, dtype=i32))


def calls(**kw):
    """Every call with operands in order, and kw in the place of the ones it names."""
    a = dict(q=z(B, T, Hq, dh), k=z(B, T, H, dh), v=z(B, T, H, dh), w=z(dh), wk=z(dh), pos=z(B, T, 3, dtype=i32), f=z(32, dtype=f32),
             ax=z(32, dtype=u8), mask=z(B, T, dtype=i32), table=z(B, W, dtype=i32), lens=z(B, dtype=i32), n_new=z(B, dtype=i32),
             R=z(H, dh, dh), parents=z(B, T, dtype=i32), tree=z(B, T, 1, dtype=i32), leaf=z(B, dtype=i32),
             bounds=z(N, H, 2, dh), visible=z(B, T, dtype=i32), sel=z(B, T, H, 7, dtype=i32), out=z(B, T, Hq, dh), qo=z(B, T, Hq, dh),
             ko=z(B, T, H, dh), new=z(B, dtype=i32), depth=z(B, T, dtype=i32), ws=z(1 << 20, dtype=u8), stream=None)
    a.update(kw)
    c = cache()
    return {
        "norm": lambda: rs.norm_rotary(a["q"], a["k"], a["w"], a["wk"], 1e-6, a["pos"], a["f"], a["ax"], out=(a["qo"], a["ko"]),
                                       stream=a["stream"]),
        "append": lambda: rs.append_rotary(c, a["k"], a["v"], a["mask"], a["table"], a["lens"], a["pos"], a["f"], a["ax"], a["R"],
                                           a["q"], a["w"], a["wk"], n_new=a["n_new"], q_out=a["qo"], stream=a["stream"]),
        "masks": lambda: rs.tree_masks(a["parents"], out=(a["tree"], a["depth"]), stream=a["stream"]),
        "tree": lambda: rs.attend_tree(a["q"], c, a["table"], a["lens"], a["tree"], a["R"], a["n_new"], workspace=a["ws"], out=a["out"],
                                       stream=a["stream"]),
        "accept": lambda: rs.cache_accept(c, a["table"], a["lens"], a["tree"], a["leaf"], a["new"], stream=a["stream"]),
        "bounds": lambda: rs.page_bounds(c, a["table"], a["lens"], a["bounds"], 1, stream=a["stream"]),
        "select": lambda: rs.select_pages(a["q"], c, a["bounds"], a["table"], a["lens"], 7, visible=a["visible"], workspace=a["ws"],
                                          out=a["sel"], stream=a["stream"]),
        "selected": lambda: rs.attend_selected(a["q"], c, a["table"], a["lens"], a["sel"], a["R"], visible=a["visible"],
                                               workspace=a["ws"], out=a["out"], stream=a["stream"]),
    }


USED = {
    "norm": "q k w wk pos f ax qo ko", "append": "q k v w wk pos f ax mask table lens n_new R qo", "masks": "parents tree depth",
    "tree": "q table lens n_new tree R out", "accept": "table lens tree leaf new", "bounds": "table lens bounds",
    "select": "q table lens visible bounds sel", "selected": "q table lens visible sel R out",
}


@pytest.mark.parametrize("name", USED)
def test_shapes_and_types_are_checked(name):
    with pytest.raises(ValueError, match="device tensors only"):
        calls()[name]()
    good = dict(q=(B, T, Hq, dh), k=(B, T, H, dh), v=(B, T, H, dh), w=(dh,), wk=(dh,), pos=(B, T, 3), f=(32,), ax=(32,), mask=(B, T),
                table=(B, W), lens=(B,), n_new=(B,), R=(H, dh, dh), parents=(B, T), tree=(B, T, 1), leaf=(B,),
                bounds=(N, H, 2, dh), visible=(B, T), sel=(B, T, H, 7), out=(B, T, Hq, dh), qo=(B, T, Hq, dh), ko=(B, T, H, dh),
                new=(B,), depth=(B, T))
    for x in USED[name].split():
        dt = {"f": f32, "ax": u8}.get(x, i32 if x in ("pos mask table lens n_new parents tree leaf visible sel new depth").split() else bf)
        free = {"table": 1, "f": 0, "sel": 3 if name == "selected" else None, "pos": 2, "q": 2, "tree": 1 if name == "accept" else None}  # sizes that a call takes from it
        for d in range(len(good[x])):
            bad = list(good[x])
            bad[d] += 1
            if free.get(x) == d:
                continue
            with pytest.raises((ValueError, TypeError)) as e:
                calls(**{x: z(*bad, dtype=dt)})[name]()
            assert "device tensors only" not in str(e.value), (x, d)
        with pytest.raises((ValueError, TypeError)) as e:
            calls(**{x: z(*good[x], dtype=torch.float64)})[name]()
        assert "device tensors only" not in str(e.value), x
        with pytest.raises((ValueError, TypeError, AttributeError)):
            calls(**{x: [1, 2]})[name]()


def test_one_tree_for_all_and_optional_operands():
    for name, kw in (("tree", dict(tree=z(1, T, 1, dtype=i32))), ("accept", dict(tree=z(1, T, 1, dtype=i32))),
                     ("tree", dict(R=None, n_new=None)), ("append", dict(R=None, n_new=None, ax=None, w=None, wk=None)),
                     ("append", dict(q=None, w=None, qo=None)), ("append", dict(pos=z(B, T, dtype=i32))), ("norm", dict(q=None)),
                     ("norm", dict(k=None)), ("masks", dict(depth=None)), ("selected", dict(visible=None, R=None)),
                     ("select", dict(visible=None)), ("tree", dict(out=z(B, T, Hq, dh, dtype=f32)))):
        with pytest.raises(ValueError, match="device tensors only"):
            calls(**kw)[name]()
    with pytest.raises(ValueError, match="both None"):
        calls(q=None, k=None)["norm"]()
    with pytest.raises(ValueError, match="need q"):
        calls(q=None, w=z(dh), qo=None)["append"]()
    with pytest.raises(ValueError, match="one stride"):
        calls(q=z(1, 1, Hq, dh).expand(B, T, Hq, dh))["tree"]()
    for x in ("k", "v", "q"):
        with pytest.raises(ValueError, match="one stride"):
            calls(**{x: z(1, 1, H if x != "q" else Hq, dh).expand(B, T, H if x != "q" else Hq, dh)})["append"]()


@pytest.mark.parametrize("name", USED)
def test_calls_allocate_on_their_stream(monkeypatch, name):
    none = dict(qo=None, ko=None, out=None, new=None, ws=None)
    if name == "select":
        none["sel"] = None
    run = {"masks": lambda s: rs.tree_masks(z(B, T, dtype=i32), stream=s),
           "norm": lambda s: rs.norm_rotary(z(B, T, Hq, dh), z(B, T, H, dh), None, None, 1e-6, z(B, T, dtype=i32), z(32, dtype=f32), stream=s)}
    call = run.get(name, lambda s: calls(**none, stream=s)[name]())
    # (what this test makes itself is not counted: it is made before)
    if name not in run:
        made = calls(**none, stream=None)  # noqa: F841
    got = allocations(monkeypatch, call)
    assert all(got) and (got or name == "bounds")


# ---- the library's refusals --------------------------------------------------

def lib_calls():
    """Each call of the C ABI with good arguments; changes by name. What passes the checks
    reaches a launch, which finds no device."""
    lib, A = rs.load(), ctypes.c_void_p
    base = dict(K=0x10000000, V=0x20000000, mask=0x30000000, slot=0x31000000, q=0x40000000, k=0x41000000, v=0x42000000, R=0x43000000,
                wq=0x44000000, wk=0x44100000, pos=0x45000000, f=0x45100000, ax=0x45200000, nm=0x46000000, table=0x50000000,
                lens=0x51000000, n_new=0x52000000, visible=0x53000000, tree=0x54000000, parents=0x55000000, leaf=0x56000000,
                bounds=0x57000000, qo=0x60000000, ko=0x61000000, out=0x62000000, sel=0x63000000, new=0x64000000, depth=0x65000000,
                ws=0x80000000)
    size = dict(B=3, T=2, Hq=4, H=2, dh=64, G=8, page=16, n_pages=5, vcap=64, W=60, dtype=rs.BF16, odt=rs.BF16, eps=1e-6, axes=3,
                pairs=32, n_sel=40, first=1, recent=2, max_len=0, trees=3, scale=0.0, qs=0, ks=0, vs=0, wsb=1 << 26, Tb=1)

    def run(name, **kw):
        v = {**base, **size, **kw}
        p = {x: A(v[x]) if v[x] is not None else None for x in base}
        d = ctypes.byref(rs.PagesDesc(v["n_pages"], v["page"], v["vcap"], v["H"], v["dh"], v["G"], p["K"], p["V"], p["mask"], p["slot"]))
        s = None
        st = {
            "norm": lambda: lib.rolesub_norm_rotary(v["B"], v["T"], v["Hq"], v["H"], v["dh"], v["dtype"], p["q"], v["qs"], p["k"], v["ks"],
                                                    p["wq"], p["wk"], v["eps"], p["pos"], v["axes"], p["f"], p["ax"], v["pairs"], 0,
                                                    p["qo"], p["ko"], s),
            "append": lambda: lib.rolesub_append_rotary(d, v["dtype"], v["B"], v["T"], v["Hq"], p["q"], v["qs"], p["k"], v["ks"], p["v"],
                                                        v["vs"], p["R"], p["nm"], p["wq"], p["wk"], v["eps"], p["pos"], v["axes"],
                                                        p["f"], p["ax"], v["pairs"], 0, p["table"], v["W"], p["lens"], p["n_new"],
                                                        p["qo"], s),
            "masks": lambda: lib.rolesub_tree_masks(v["B"], v["T"], p["parents"], p["tree"], p["depth"], s),
            "tree": lambda: lib.rolesub_attend_tree(d, v["dtype"], v["B"], v["Hq"], v["T"], p["q"], v["qs"], p["table"], v["W"], p["lens"],
                                                    p["n_new"], p["tree"], v["trees"], v["max_len"], p["R"], v["scale"], p["out"],
                                                    v["odt"], p["ws"], v["wsb"], s),
            "accept": lambda: lib.rolesub_cache_accept(d, v["dtype"], v["B"], v["T"], p["table"], v["W"], p["lens"], p["tree"], v["trees"],
                                                       p["leaf"], p["new"], s),
            "bounds": lambda: lib.rolesub_page_bounds(d, v["dtype"], v["B"], v["Tb"], p["table"], v["W"], p["lens"], p["bounds"], s),
            "select": lambda: lib.rolesub_select_pages(d, v["dtype"], v["B"], v["Hq"], v["T"], p["q"], v["qs"], p["bounds"], p["table"],
                                                       v["W"], p["lens"], p["visible"], v["max_len"], v["n_sel"], v["first"],
                                                       v["recent"], p["sel"], p["ws"], v["wsb"], s),
            "selected": lambda: lib.rolesub_attend_selected(d, v["dtype"], v["B"], v["Hq"], v["T"], p["q"], v["qs"], p["table"], v["W"],
                                                            p["lens"], p["visible"], p["sel"], v["n_sel"], p["R"], v["scale"], p["out"],
                                                            v["odt"], p["ws"], v["wsb"], s),
        }[name]()
        return st, lib.rolesub_last_error().decode()
    return base, run


INVALID, UNSUPPORTED, HIP = 1, 2, 4
PAGED = [x for x in USED if x not in ("norm", "masks")]


def _no_gpu():
    if torch.cuda.is_available():
        pytest.skip("calls that pass the checks would be launched")


@pytest.mark.parametrize("name", USED)
def test_good_calls_reach_the_launch(name):
    _no_gpu()
    st, why = lib_calls()[1](name)
    assert st == HIP, why


REFUSED = {
    "norm append": [(dict(dtype=7), UNSUPPORTED), (dict(dh=96), UNSUPPORTED), (dict(B=-1), INVALID), (dict(T=-1), INVALID),
                    (dict(pairs=0), INVALID), (dict(pairs=33), INVALID), (dict(axes=0), UNSUPPORTED), (dict(axes=9), UNSUPPORTED),
                    (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
                    (dict(Hq=0), INVALID), (dict(pos=None), INVALID), (dict(f=None), INVALID), (dict(qo=None), INVALID),
                    (dict(q=0x40000008), UNSUPPORTED), (dict(k=0x41000008), UNSUPPORTED), (dict(qo=0x60000004), UNSUPPORTED),
                    (dict(qs=8), INVALID), (dict(ks=129), UNSUPPORTED), (dict(B=1 << 20, T=1 << 11), UNSUPPORTED),
                    (dict(Hq=65535), UNSUPPORTED)],
    "norm": [(dict(q=None, k=None), INVALID), (dict(ko=None), INVALID), (dict(H=0), INVALID), (dict(ko=0x61000008), UNSUPPORTED)],
    "append": [(dict(nm=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(table=None), INVALID),
               (dict(lens=None), INVALID), (dict(v=0x42000008), UNSUPPORTED), (dict(vs=130), UNSUPPORTED), (dict(R=0x43000008), UNSUPPORTED),
               (dict(W=-1), INVALID)],
    "masks": [(dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(T=257), UNSUPPORTED), (dict(parents=None), INVALID), (dict(tree=None), INVALID),
              (dict(B=1 << 24), UNSUPPORTED)],
    "tree selected": [(dict(odt=5), UNSUPPORTED), (dict(dtype=rs.F32, odt=rs.BF16), UNSUPPORTED), (dict(B=-1), INVALID), (dict(T=-1), INVALID),
                      (dict(W=-1), INVALID), (dict(Hq=3), INVALID), (dict(Hq=0), INVALID), (dict(scale=float("nan")), INVALID),
                      (dict(scale=float("inf")), INVALID), (dict(q=None), INVALID), (dict(lens=None), INVALID), (dict(out=None), INVALID),
                      (dict(table=None), INVALID), (dict(out=0x62000008), UNSUPPORTED), (dict(R=0x43000002), UNSUPPORTED),
                      (dict(qs=100), INVALID), (dict(qs=257), UNSUPPORTED), (dict(wsb=16), INVALID), (dict(ws=None), INVALID),
                      (dict(ws=0x80000008), INVALID), (dict(B=1 << 24, trees=1, wsb=1 << 62), UNSUPPORTED)],
    "tree": [(dict(tree=None), INVALID), (dict(T=257), UNSUPPORTED), (dict(trees=2), INVALID), (dict(trees=0), INVALID), (dict(max_len=-1), INVALID),
             (dict(W=1 << 27), UNSUPPORTED)],
    "accept": [(dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(T=257), UNSUPPORTED), (dict(W=-1), INVALID), (dict(trees=2), INVALID),
               (dict(tree=None), INVALID), (dict(leaf=None), INVALID), (dict(lens=None), INVALID), (dict(table=None), INVALID),
               (dict(B=1 << 24, trees=1), UNSUPPORTED)],
    "bounds": [(dict(B=-1), INVALID), (dict(Tb=-1), INVALID), (dict(W=-1), INVALID), (dict(table=None), INVALID), (dict(lens=None), INVALID),
               (dict(bounds=None), INVALID), (dict(bounds=0x57000008), UNSUPPORTED), (dict(B=1 << 26), UNSUPPORTED)],
    "select": [(dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(W=-1), INVALID), (dict(max_len=-1), INVALID), (dict(Hq=3), INVALID),
               (dict(n_sel=0), INVALID), (dict(first=-1), INVALID), (dict(recent=-1), INVALID), (dict(first=30, recent=11), INVALID),
               (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), INVALID), (dict(q=None), INVALID), (dict(lens=None), INVALID), (dict(sel=None), INVALID),
               (dict(table=None), INVALID), (dict(bounds=None), INVALID), (dict(bounds=0x57000008), UNSUPPORTED), (dict(qs=5), INVALID),
               (dict(wsb=64), INVALID), (dict(ws=None), INVALID), (dict(ws=0x80000008), INVALID), (dict(W=1 << 27), UNSUPPORTED),
               (dict(B=1 << 24, wsb=1 << 62), UNSUPPORTED)],
    "selected": [(dict(sel=None), INVALID), (dict(n_sel=0), INVALID), (dict(n_sel=(1 << 26) + 1), UNSUPPORTED), (dict(W=(1 << 26) + 1), UNSUPPORTED)],
}


@pytest.mark.parametrize("names,kw,want", [(n, kw, st) for n, x in REFUSED.items() for kw, st in x])
def test_refusals(names, kw, want):
    _no_gpu()
    for name in names.split():
        st, why = lib_calls()[1](name, **kw)
        assert st == want and f"rolesub_{dict(norm='norm_rotary', append='append_rotary').get(name, '')}" in why, (name, kw, st, why)


@pytest.mark.parametrize("name", PAGED)
def test_caches_are_checked(name):
    _no_gpu()
    run = lib_calls()[1]
    for kw in (dict(page=24), dict(page=512), dict(dh=32), dict(G=33), dict(n_pages=1 << 26)):
        assert run(name, **kw)[0] == UNSUPPORTED, kw
    for kw in (dict(n_pages=-1), dict(vcap=-1), dict(H=0), dict(G=7), dict(K=None), dict(V=None), dict(mask=None), dict(slot=None)):
        assert run(name, **kw)[0] == INVALID, kw


OVERLAPS = {  # outputs (the cache too where it is written), and what each must lie apart from
    "norm": ("qo ko", "q k wq wk pos f ax"),
    "append": ("qo K V mask slot", "q k v R wq wk pos f ax nm table lens n_new"),
    "masks": ("tree depth", "parents"),
    "tree": ("out ws", "q R K V mask slot table lens n_new tree"),
    "accept": ("new K V mask slot", "table lens tree leaf"),
    "bounds": ("bounds", "K V mask slot table lens"),
    "select": ("sel ws", "q bounds table lens visible K V mask slot"),
    "selected": ("out ws", "q R K V mask slot table lens visible sel"),
}


@pytest.mark.parametrize("name", OVERLAPS)
def test_operands_that_overlap_are_refused(name):
    _no_gpu()
    base, run = lib_calls()
    outs, ins = (x.split() for x in OVERLAPS[name])
    inside = {"out": {"q"}, "qo": {"q"}, "ko": {"k"}}  # an input's own place is allowed
    for o in outs:
        for x in ins + [y for y in outs if y != o and not (o in "KVmaskslot" and y in "KVmaskslot")]:
            if x in inside.get(o, ()):
                assert run(name, **{o: base[x]})[0] == HIP, (o, x)
                st, why = run(name, **{o: base[x] + 16})
            else:
                st, why = run(name, **{x: base[o]} if o in ("K", "V", "mask", "slot") else {o: base[x]})
            assert st == INVALID and "overlap" in why, (o, x, st, why)


def test_parts_of_a_fused_projection_are_allowed():
    """q turned in place while k and v lie between its rows."""
    _no_gpu()
    base, run = lib_calls()
    row = (4 + 2 + 2) * 64
    kw = dict(q=base["q"], k=base["q"] + 4 * 64 * 2, v=base["q"] + 6 * 64 * 2, qo=base["q"], qs=row, ks=row, vs=row)
    assert run("append", **kw)[0] == HIP
    assert run("append", **{**kw, "v": base["q"] + 3 * 64 * 2})[0] == INVALID
    assert run("append", **{**kw, "qo": base["q"] + 4 * 64 * 2})[0] == INVALID
    n = dict(q=kw["q"], k=kw["k"], qo=kw["q"], ko=kw["k"], qs=row, ks=row)
    assert run("norm", **n)[0] == HIP
    assert run("norm", **{**n, "ko": kw["q"] + 2 * 64 * 2})[0] == INVALID


def test_empty_calls_do_nothing():
    run = lib_calls()[1]
    for name in USED:
        assert run(name, B=0)[0] == 0, name
    for name in ("norm", "append", "masks", "tree", "select", "selected"):
        assert run(name, T=0)[0] == 0, name
    assert run("bounds", Tb=0)[0] == 0 and run("bounds", W=0)[0] == 0


def test_workspaces_grow_with_the_call():
    lib = rs.load()
    d = ctypes.byref(rs.PagesDesc(9, 16, 64, 4, 128, 8, None, None, None, None))
    sizes = (1, 2, 3, 7, 16, 33, 64, 100)
    for ask in (lambda b, t, n: lib.rolesub_attend_tree_workspace_size(d, b, 16, t, 37 * n),
                lambda b, t, n: lib.rolesub_select_pages_workspace_size(d, b, t, 5003 * n),
                lambda b, t, n: lib.rolesub_attend_selected_workspace_size(d, b, 16, t, n)):
        last = {}
        for x in sizes:
            for a in (1, 5, 40):
                now = ask(x, a, 9), ask(a, x, 9), ask(a, 3, x)
                assert all(p <= q for p, q in zip(last.get(a, now), now)), (x, a)
                last[a] = now
    assert lib.rolesub_attend_tree_workspace_size(None, 1, 16, 1, 9) == lib.rolesub_select_pages_workspace_size(None, 1, 1, 9) == 0


@pytest.mark.parametrize("name", ["tree", "selected"])
@pytest.mark.parametrize("H", [1, 8])
def test_a_workspace_serves_every_smaller_call(name, H):
    _no_gpu()
    lib, run = rs.load(), lib_calls()[1]
    d = ctypes.byref(rs.PagesDesc(9, 64, 64, H, 64, 8, None, None, None, None))
    need, ask = {}, {}
    for B in (1, 5, 65, 300):
        for Tq in (1, 4, 8, 15, 16, 17, 20, 24, 32, 33, 40, 64, 65, 96, 129, 250):
            for n in (1, 9, 300, 2100):  # pages of 64 tokens
                ask[B, Tq, n] = (lib.rolesub_attend_tree_workspace_size(d, B, H, Tq, 64 * n) if name == "tree" else
                                 lib.rolesub_attend_selected_workspace_size(d, B, H, Tq, n))
                # far apart: the operands of no call overlap, and the refusal comes before a launch
                kw = {x: (i + 1) << 44 for i, x in enumerate(lib_calls()[0])}
                st, why = run(name, **{**kw, "ws": None}, B=B, T=Tq, Hq=H, H=H, page=64, W=2100, max_len=64 * n, n_sel=n, trees=1, wsb=0)
                got = re.search(r"workspace of (\d+) bytes", why) if st == INVALID else None
                assert got or st == HIP, why
                need[B, Tq, n] = int(got.group(1)) if got else 0
    for x, y in need.items():
        for z_, most in ask.items():
            if all(i <= j for i, j in zip(x, z_)):
                assert y <= most, (x, y, z_, most)


# ---- layers ------------------------------------------------------------------

def test_layers_refuse_before_anything_runs():
    from paper_2608_18410_amd.pipeline import decode_layer, draft_layer
    for kw, why in ((dict(n_sel=4, bounds=1, mass=1), "no weight"), (dict(n_sel=4), "needs bounds"), (dict(q_weight=1), "need positions"),
                    (dict(k_weight=1), "need positions")):
        with pytest.raises(ValueError, match=why):
            decode_layer(*[None] * 12, **kw)
    for kw in (dict(q_weight=1), dict(k_weight=1)):
        with pytest.raises(ValueError, match="need positions"):
            draft_layer(*[None] * 12, **kw)


@pytest.mark.parametrize("stream", [None, "side"])
def test_layers_calls_and_streams(monkeypatch, stream):
    """Which calls a layer makes, all with the chain's stream current, and whose its outputs are."""
    from paper_2608_18410_amd import pipeline
    made, marked, now = [], [], ["caller"]

    class Out:
        is_cuda, device, shape = True, "cuda:0", (2, 5)

        def record_stream(self, s):
            marked.append(s)

    class On:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            now.append(self.s)

        def __exit__(self, *a):
            now.pop()

    def call(name, out):
        return lambda *a, **kw: (made.append((name, now[-1])), out)[1]

    monkeypatch.setattr(pipeline.torch.cuda, "stream", On)
    monkeypatch.setattr(pipeline.torch.cuda, "current_stream", lambda d=None: now[-1])
    for name in ("append_rotary", "attend_paged", "attend_tree", "attend_selected", "cache_accept", "page_bounds", "select_pages",
                 "rotate_values", "cache_append"):
        monkeypatch.setattr(pipeline.rs, name, call(name, Out()))
    monkeypatch.setattr(pipeline.rs, "route", call("route", {"mask": None}))
    at = "caller" if stream is None else stream
    tree = torch.zeros(2, 5, 1)
    for run, want in (
            (lambda: pipeline.decode_layer(*[None] * 12, positions=1, stream=stream), ["route", "append_rotary", "attend_paged"]),
            (lambda: pipeline.decode_layer(*[None] * 12, positions=1, n_sel=3, bounds=1, stream=stream),
             ["route", "append_rotary", "page_bounds", "select_pages", "attend_selected"]),
            (lambda: pipeline.draft_layer(*[None] * 12, positions=1, stream=stream), ["route", "append_rotary", "attend_tree"]),
            (lambda: pipeline.draft_layer(*[None] * 12, n_new=1, stream=stream), ["route", "rotate_values", "cache_append", "attend_tree"]),
            (lambda: pipeline.accept_layer(None, None, None, tree, None, stream=stream), ["cache_accept"]),
            (lambda: pipeline.accept_layer(None, None, None, tree, None, bounds=1, stream=stream), ["cache_accept", "page_bounds"])):
        made.clear()
        marked.clear()
        run()
        assert made == [(x, at) for x in want] and marked == ([] if stream is None else ["caller"])


# ---- the assembly ------------------------------------------------------------

@pytest.mark.skipif(not shutil.which(build.HIPCC), reason="needs hipcc")
@pytest.mark.parametrize("src", ["k_tree.hip", "k_listed.hip", "k_norm.hip"])
def test_no_product_is_read_early(tmp_path, src):
    out = str(tmp_path / "k.s")
    r = subprocess.run([build.HIPCC, *build.FLAGS, "-S", "--offload-device-only", os.path.join(build.CSRC, src), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    n = 0
    for name, ins, labels in functions(open(out).read()):
        n += sum(op.startswith("v_mfma") for op, _ in ins)
        assert not list(early_reads(ins, labels)), name
    assert n > 100
