"""decode_layer and evict_layer without a GPU: what they refuse before anything is written,
and calls of the C ABI on empty inputs."""
import ctypes

import pytest
import torch

import paper_2608_18410_amd as rs
from paper_2608_18410_amd import pipeline

i32 = torch.int32


@pytest.fixture
def calls(monkeypatch):
    """The library's calls recorded, their outputs plain tensors."""
    done = []

    def evict_tokens(mass, lens, keep, *a, **kw):
        done.append("evict_tokens")
        return torch.zeros((mass.shape[0], keep), dtype=i32), torch.zeros(mass.shape[0], dtype=i32)

    def cache_compact(src, table, idx, n, dst, dst_table, mass, mass_out):
        done.append("cache_compact")
        if mass.data_ptr() == mass_out.data_ptr():
            raise rs.RolesubError("rolesub_cache_compact", 1, "mass_in and mass_out overlap")
        return mass_out

    monkeypatch.setattr(pipeline.rs, "evict_tokens", evict_tokens)
    monkeypatch.setattr(pipeline.rs, "cache_compact", cache_compact)
    return done


def test_evict_layer_refuses_before_it_clears_weights(calls):
    base = torch.rand(3 * 40)
    mass = base[:80].view(2, 40)
    kept = base.clone()
    go = lambda out, m=mass: pipeline.evict_layer(None, None, None, m, 8, 0, 0, None, None, mass_out=out)  # noqa: E731
    for bad in (mass, base[40:].view(2, 40), base[72:120].view(2, 24), base[:80].view(2, 40)[:, :8], torch.rand(2, 7),
                torch.rand(3, 8), torch.rand(2, 8, 1), torch.rand(2, 8, dtype=torch.float64), torch.rand(8, 2).T):
        with pytest.raises(ValueError):
            go(bad)
        assert torch.equal(base, kept) and not calls
    out = go(base[80:].view(2, 20))[1]
    assert not out.any() and torch.equal(base[:80], kept[:80]) and calls == ["evict_tokens", "cache_compact"]
    assert go(None)[1].shape == (2, 40)


def test_layers_mark_their_outputs_for_the_callers_stream(monkeypatch):
    """What is allocated on the chain's stream goes on with the caller's."""
    marked, now = [], ["caller"]

    class Out:
        is_cuda, device, shape = True, "cuda:0", (2, 40)

        def __init__(self, name):
            self.name = name

        def record_stream(self, s):
            marked.append((self.name, s))

        def zero_(self):
            pass

    class On:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            now.append(self.s)

        def __exit__(self, *a):
            now.pop()

    monkeypatch.setattr(pipeline.torch.cuda, "stream", On)
    monkeypatch.setattr(pipeline.torch.cuda, "current_stream", lambda d=None: now[-1])
    monkeypatch.setattr(pipeline.torch, "empty_like", lambda t: Out("mass"))
    monkeypatch.setattr(pipeline.rs, "route", lambda *a, **kw: {"mask": None})
    monkeypatch.setattr(pipeline.rs, "rotate_values", lambda *a, **kw: None)
    monkeypatch.setattr(pipeline.rs, "cache_append", lambda *a, **kw: None)
    monkeypatch.setattr(pipeline.rs, "attend_paged", lambda *a, **kw: Out("out"))
    monkeypatch.setattr(pipeline.rs, "evict_tokens", lambda *a, **kw: (Out("idx"), Out("n")))
    monkeypatch.setattr(pipeline.rs, "cache_compact", lambda *a, **kw: None)
    for stream in (None, "side"):
        pipeline.decode_layer(*[None] * 12, stream=stream)
        pipeline.evict_layer(None, None, None, Out("old"), 8, 0, 0, None, None, stream=stream)
        assert marked == ([] if stream is None else [(x, "caller") for x in ("out", "n", "mass", "idx")])


def test_expanded_operands_are_refused():
    """One token for many, without its own memory: not rows at a stride."""
    bf = torch.bfloat16
    z = lambda *s, dtype=bf: torch.zeros(s, dtype=dtype)  # noqa: E731
    f = z(32, dtype=torch.float32)
    cache = rs.PagedCache(K=z(5, 2, 16, 64), V=z(5, 2, 64, 8), mask=z(5, 16, dtype=i32), slot=z(5, 16, dtype=i32))
    for B, T in ((3, 1), (1, 3), (3, 2)):
        table, lens = z(B, 2, dtype=i32), z(B, dtype=i32)
        x, ok = z(1, 1, 2, 64).expand(B, T, 2, 64), z(B, T, 2, 64)
        for call in (lambda: rs.rotary(x, None, z(B, T, dtype=i32), f), lambda: rs.rotary(ok, x, z(B, T, dtype=i32), f),
                     lambda: rs.rotary(ok, None, z(B, T, dtype=i32), f, out=(x, None)),
                     lambda: rs.attend_paged(x, cache, table, lens),
                     lambda: rs.cache_append(cache, x, ok, z(B, T, dtype=i32), table, lens),
                     lambda: rs.cache_append(cache, ok, x, z(B, T, dtype=i32), table, lens)):
            with pytest.raises(ValueError, match="one stride"):
                call()
    one = torch.zeros(9, 2, 64, dtype=bf)[4].expand(1, 1, 2, 64)  # a single token is its own memory
    with pytest.raises(ValueError, match="device tensors only"):
        rs.rotary(one, None, z(1, 1, dtype=i32), f)


def test_an_empty_table_needs_no_workspace_for_weights():
    """The smallest calls: no page a sequence. What the size query answers is enough; here the
    launch that follows finds no device, on the GPU the outputs are zeros."""
    lib, a = rs.load(), ctypes.c_void_p(0x10000000)
    for mp, ml in ((0, 0), (0, 7)):
        pg = rs.PagesDesc(5, 16, 64, 2, 64, 8, a, a, a, a)
        need = lib.rolesub_attend_paged_workspace_size(ctypes.byref(pg), 3, 4, 1, 0, 1)
        assert need == 0
        if torch.cuda.is_available():
            continue
        st = lib.rolesub_attend_paged(ctypes.byref(pg), rs.BF16, 3, 4, 1, a, 0, None, mp, a, None, ml, None, 0.0,
                                      ctypes.c_void_p(0x20000000), rs.BF16, None, 1.0, ctypes.c_void_p(0x30000000), 0, None, 0,
                                      None)
        assert "workspace" not in lib.rolesub_last_error().decode() and st != 1


def test_attend_paged_refuses_operands_that_overlap():
    lib = rs.load()
    P = ctypes.c_void_p
    base = dict(K=0x10000000, V=0x20000000, mask=0x30000000, slot=0x31000000, q=0x40000000, table=0x50000000, lens=0x51000000,
                visible=0x52000000, R=0x53000000, out=0x60000000, mi=0x70000000, mo=0x70000000, ws=0x80000000)
    dense = 3 * 2 * 4 * 64 * 2

    def call(qs=0, odt=rs.BF16, **kw):
        a = {k: P(v) for k, v in {**base, **kw}.items()}
        pg = rs.PagesDesc(5, 16, 64, 2, 64, 8, a["K"], a["V"], a["mask"], a["slot"])
        need = lib.rolesub_attend_paged_workspace_size(ctypes.byref(pg), 3, 4, 2, 320, 1)
        st = lib.rolesub_attend_paged(ctypes.byref(pg), rs.BF16, 3, 4, 2, a["q"], qs, a["table"], 20, a["lens"], a["visible"], 0,
                                      a["R"], 0.0, a["out"], odt, a["mi"], 1.0, a["mo"], 320, a["ws"], need, None)
        return st, lib.rolesub_last_error().decode()

    if torch.cuda.is_available():
        pytest.skip("calls that pass the checks would be launched")
    for out in ("out", "mo", "ws"):
        for x, v in base.items():
            if x == out or {x, out} == {"mi", "mo"}:
                continue
            kw = {out: v, **({"mi": v} if out == "mo" and x != "mi" else {})}
            if (out, x) != ("out", "q"):
                st, why = call(**kw)
                assert st == 1 and "overlap" in why, (out, x, why)
    assert call(mo=base["mi"] + 64)[0] == 1
    assert call(out=base["q"] + 16)[0] == 1 and call(out=base["q"] + dense - 16)[0] == 1
    assert call(out=base["q"], odt=rs.F32)[0] == 1 and call(out=base["q"], qs=512)[0] == 1
    for kw in ({}, dict(out=base["q"]), dict(out=base["q"] + dense), dict(out=base["q"] - dense), dict(mi=base["mi"] + 3 * 320 * 4)):
        st, why = call(**kw)  # what is allowed comes as far as the launch, which finds no device
        assert st == 4 and "overlap" not in why, (kw, why)


def test_evict_refuses_operands_that_overlap():
    """The new lengths in the old ones' place, for one: other workgroups still read those."""
    lib, P = rs.load(), ctypes.c_void_p
    base = dict(mass=0x10000000, lens=0x20000000, idx=0x30000000, n=0x40000000, ws=0x50000000)

    def call(**kw):
        a = {k: P(v) for k, v in {**base, **kw}.items()}
        need = lib.rolesub_evict_workspace_size(3, 40000)
        st = lib.rolesub_evict_tokens(3, 40000, a["mass"], 40000, a["lens"], 8, 1, 2, a["idx"], a["n"], a["ws"], need, None)
        return st, lib.rolesub_last_error().decode()

    if torch.cuda.is_available():
        pytest.skip("calls that pass the checks would be launched")
    for out in ("idx", "n", "ws"):
        for x, v in base.items():
            if x != out:
                st, why = call(**{out: v})
                assert st == 1 and "overlap" in why, (out, x, why)
    assert call(n=base["lens"] + 8)[0] == 1 and call(idx=base["mass"] + 3 * 40000 * 4 - 4)[0] == 1
    for kw in ({}, dict(n=base["lens"] + 12), dict(idx=base["mass"] + 3 * 40000 * 4)):
        st, why = call(**kw)
        assert st == 4 and "overlap" not in why, (kw, why)


def test_append_and_compact_refuse_lengths_and_tables_inside_the_cache():
    lib, P = rs.load(), ctypes.c_void_p
    if torch.cuda.is_available():
        pytest.skip("calls that pass the checks would be launched")
    K, V, M, S = 0x10000000, 0x20000000, 0x30000000, 0x31000000
    inside = (K, K + 5 * 2 * 16 * 64 * 2 - 4, V, V + 5 * 2 * 64 * 8 * 2 - 4, M, M + 5 * 16 * 4 - 4, S, S + 5 * 16 * 4 - 4)
    pg = ctypes.byref(rs.PagesDesc(5, 16, 64, 2, 64, 8, *map(P, (K, V, M, S))))
    other = ctypes.byref(rs.PagesDesc(5, 16, 64, 2, 64, 8, *map(P, (0x41000000, 0x42000000, 0x43000000, 0x44000000))))

    def append(mask=0x50000000, table=0x51000000, lens=0x52000000, n=0x53000000, k=0x54000000):
        st = lib.rolesub_cache_append(pg, rs.BF16, 2, 3, P(k), 0, P(0x55000000), 0, P(mask), P(table), 2, P(lens), P(n), None)
        return st, lib.rolesub_last_error().decode()

    def compact(src=other, idx=0x50000000, n=0x51000000, table=0x52000000, dt=0x53000000, mi=0x54000000, mo=0x55000000):
        st = lib.rolesub_cache_compact(src, pg, rs.BF16, 2, P(table), 2, P(idx), P(n), 4, P(dt), 2, P(mi), 40, P(mo), 9, None)
        return st, lib.rolesub_last_error().decode()

    for call, names in ((append, ("mask", "table", "lens", "n")), (compact, ("idx", "n", "table", "dt", "mi", "mo"))):
        for name in names:
            for at in inside:
                st, why = call(**{name: at})
                assert st == 1 and "overlaps" in why, (call, name, hex(at), why)
    for name, at in (("idx", 0x55000000), ("n", 0x55000008), ("table", 0x55000000 + 4 * 12), ("dt", 0x55000000 - 12)):
        assert compact(**{name: at})[0] == 1, name
    # keys of other pages are no matter of the host's, and src may be dst
    for st, why in (append(), append(k=K), compact(), compact(src=pg), compact(table=0x55000000 + 4 * 13)):
        assert st == 4 and "overlap" not in why, why
