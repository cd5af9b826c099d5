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
