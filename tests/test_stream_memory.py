"""Memory that a call with stream= allocates by itself comes out of that stream's pool: a
block of the current stream's may still be in use there, which the call's stream does
not wait for. Without a GPU: where each allocation happens, up to the device check."""
import contextlib

import pytest
import torch

import paper_2608_18410_amd as rs
from paper_2608_18410_amd import rolesub

bf, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def z(*shape, dtype=bf):
    return torch.zeros(shape, dtype=dtype)


class Stream:
    device_index, cuda_stream = 0, 0


def _cache():
    return rs.PagedCache(K=z(5, 2, 16, 64), V=z(5, 2, 64, 8), mask=z(5, 16, dtype=i32), slot=z(5, 16, dtype=i32))


PAGED = {
    "rotary": lambda s: rs.rotary(z(2, 3, 4, 64), z(2, 3, 2, 64), z(2, 3, dtype=i32), z(32, dtype=f32), stream=s),
    "attend_paged": lambda s: rs.attend_paged(z(2, 3, 4, 64), _cache(), z(2, 2, dtype=i32), z(2, dtype=i32),
                                              mass=z(2, 32, dtype=f32), stream=s),
    "evict_tokens": lambda s: rs.evict_tokens(z(2, 40, dtype=f32), z(2, dtype=i32), 8, stream=s),
    "cache_compact": lambda s: rs.cache_compact(_cache(), z(2, 2, dtype=i32), z(2, 8, dtype=i32), z(2, dtype=i32), _cache(),
                                                z(2, 2, dtype=i32), mass=z(2, 40, dtype=f32), stream=s),
}


def allocations(monkeypatch, call):
    """The stream that was current at each allocation of the call."""
    now, seen, empty, like = [None], [], torch.empty, torch.empty_like

    @contextlib.contextmanager
    def stream(s):
        now.append(s)
        yield
        now.pop()

    s = Stream()
    with monkeypatch.context() as m:
        m.setattr(rolesub.torch.cuda, "stream", stream)
        m.setattr(rolesub.torch, "empty", lambda *a, **kw: (seen.append(now[-1]), empty(*a, **kw))[1])
        m.setattr(rolesub.torch, "empty_like", lambda *a, **kw: (seen.append(now[-1]), like(*a, **kw))[1])
        with pytest.raises(ValueError, match="device tensors only"):
            call(s)
    return [x is s for x in seen]


@pytest.mark.parametrize("name", PAGED)
def test_paged_calls_allocate_on_their_stream(monkeypatch, name):
    got = allocations(monkeypatch, PAGED[name])
    assert got and all(got)


def _router():
    d, C, G, d_e, Hr = 32, 3, 8, 4, 16
    return rs.Router.mlp2(*(z(*x) for x in ((C, d), (C,), (C, d_e), (Hr, 2 * d + d_e), (Hr,), (G, Hr), (G,))))


def _prefix_calls():
    B, T, H, dh, G, S = 2, 6, 2, 64, 8, 4
    q, v, R = z(B, T, H, dh), z(B, T, H, dh), z(H, dh, dh)
    mask, off, vp = z(B, T, dtype=i32), z(B, T + 1, dtype=i32), z(B, H, T * G, dh // G)
    types, h, budget = z(B, T, dtype=u8), z(B, T, 32), rs.make_budget(rs.TOPK, (4,) * 4)
    Rw, vpw = z(H * dh, H * dh), z(B, T * S, H * dh // S)
    return {
        "rotate_values": lambda s: rs.rotate_values(v, R, stream=s),
        "route": lambda s: rs.route(types, budget, G, h=h, router=_router(), stream=s),
        "pack_kv": lambda s: rs.pack_kv(v, mask, G, T * G, stream=s),
        "rotate_pack": lambda s: rs.rotate_pack(v, R, mask, G, T * G, stream=s),
        "attend": lambda s: rs.attend(q, q, mask, off, vp, R, G, stream=s),
        "attend_causal": lambda s: rs.attend_causal(q, q, mask, off, vp, R, G, stream=s),
        "retain_tokens": lambda s: rs.retain_tokens(z(B, 9, dtype=f32), (9,), (4,), stream=s),
        "gather_tokens": lambda s: rs.gather_tokens(q, z(B, 3, dtype=i32), stream=s),
        "allocate_groups": lambda s: rs.allocate_groups(z(B, T, dtype=f32), types, (4,) * 4, G, z(B, T, G, dtype=f32), stream=s),
        "route_allocate": lambda s: rs.route_allocate(types, (4,) * 4, G, h, _router(), z(3), stream=s),
        "full_transpose": lambda s: rs.full_transpose(Rw, stream=s),
        "full_rotate_pack": lambda s: rs.full_rotate_pack(v, Rw, mask, S, T * S, stream=s),
        "full_values": lambda s: rs.full_values(Rw, mask, off, vpw, S, H, stream=s),
        "attend_values": lambda s: rs.attend_values(q, q, z(B, H, T, dh), stream=s),
    }


@pytest.mark.parametrize("name", list(_prefix_calls()))
def test_prefix_calls_allocate_on_their_stream(monkeypatch, name):
    got = allocations(monkeypatch, _prefix_calls()[name])
    assert got and all(got)
