"""The paged cache's normed heads, appends, drafted trees and chosen pages at their edges, without a GPU."""
import types

import numpy as np
import pytest
import torch

from oracle import paged as O
from paper_2608_18410_amd import pipeline


def test_oracle_bounds_of_a_shared_page_are_those_of_its_longest_sequence():
    rng = np.random.default_rng(0)
    P, H, dh = 16, 2, 8
    c = dict(K=rng.standard_normal((4, H, P, dh)))
    c["K"][:, :, 9:] *= 5
    table = np.array([[0, 1], [0, 2], [0, 1]])
    for lens, T in (([25, 5, 20], 1), ([5, 25, 20], 1), ([20, 25, 5], 10 ** 6), ([25, 25, 20], 2)):
        b = np.full((4, H, 2, dh), 7.0)
        O.page_bounds(c, table, lens, b, T)
        for s, n in enumerate(lens):  # what a page's bounds say holds for every sequence
            for i in range(max(n - T, 0) // P, -(-n // P)):
                k = c["K"][table[s, i], :, : n - i * P]
                assert (b[table[s, i], :, 0] <= k.min(1)).all() and (b[table[s, i], :, 1] >= k.max(1)).all()
        assert (b[3] == 7.0).all()


@pytest.mark.parametrize("max_len,want", [(0, [5, 40, 70]), (64, [5, 40, 70]), (41, [5, 40, 41]), (1000, [5, 40, 70]), (1, [1, 1, 1])])
def test_few_pages_are_attended_to_up_to_max_len(monkeypatch, max_len, want):
    """Pages are chosen among the tokens below max_len; one that it ends in is seen so far."""
    seen = []
    for name in ("append_rotary", "page_bounds", "select_pages"):
        monkeypatch.setattr(pipeline.rs, name, lambda *a, **kw: torch.zeros(1, 1))
    monkeypatch.setattr(pipeline.rs, "route", lambda *a, **kw: {"mask": None})
    monkeypatch.setattr(pipeline.rs, "attend_selected", lambda q, c, t, lens, *a, **kw: seen.append(lens.tolist()))
    cache = types.SimpleNamespace(page=16)
    lens = torch.tensor([5, 40, 70], dtype=torch.int32)
    pipeline.decode_layer(*[None] * 8, cache, torch.zeros(3, 9), lens - 1, lens, positions=1, n_sel=3, bounds=1, max_len=max_len)
    assert seen == [want] and lens.tolist() == [5, 40, 70]


@pytest.mark.parametrize("status,ways", [(1, 3), (2, 3), (4, 0)])
def test_what_one_pass_refuses_goes_through_the_separate_calls(monkeypatch, status, ways):
    """As operands that lie in the cache; a launch that failed is an error."""
    made = []

    def refuse(*a, **kw):
        raise pipeline.rs.RolesubError("rolesub_append_rotary", status, "K overlaps q")

    monkeypatch.setattr(pipeline.rs, "append_rotary", refuse)
    monkeypatch.setattr(pipeline.rs, "route", lambda *a, **kw: {"mask": None})
    monkeypatch.setattr(pipeline.rs, "norm_rotary", lambda *a, **kw: (made.append("norm_rotary"), ("q", "k"))[1])
    monkeypatch.setattr(pipeline.rs, "rotate_values", lambda *a, **kw: made.append("rotate_values"))
    monkeypatch.setattr(pipeline.rs, "cache_append", lambda *a, **kw: made.append("cache_append"))
    monkeypatch.setattr(pipeline.rs, "attend_paged", lambda q, *a, **kw: q)
    args = [None] * 5 + ["R"] + [None] * 6
    if ways:
        assert pipeline.decode_layer(*args, positions=1) == "q"
        assert made == ["norm_rotary", "rotate_values", "cache_append"]
    else:
        with pytest.raises(pipeline.rs.RolesubError):
            pipeline.decode_layer(*args, positions=1)
    with pytest.raises(pipeline.rs.RolesubError):
        pipeline.decode_layer(*[None] * 12, positions=1)


@pytest.mark.parametrize("have,max_len", [(None, 0), (99, 0), (100, 0), (500, 0), (99, 41), (100, 41)])
def test_a_layer_over_few_pages_gives_both_calls_its_workspace(monkeypatch, have, max_len):
    """Where it is large enough for the choice: a smaller one serves the attention, as it did."""
    got, asked = [], []
    q = torch.zeros(3, 2, 4, 8)
    monkeypatch.setattr(pipeline.rs, "route", lambda *a, **kw: {"mask": None})
    monkeypatch.setattr(pipeline.rs, "append_rotary", lambda *a, **kw: q)
    monkeypatch.setattr(pipeline.rs, "page_bounds", lambda *a, **kw: None)
    monkeypatch.setattr(pipeline.rs, "select_pages_workspace_size", lambda cache, *a: (asked.append(a), 100)[1])
    for name in ("select_pages", "attend_selected"):
        monkeypatch.setattr(pipeline.rs, name, lambda *a, workspace=None, **kw: (got.append(workspace), torch.zeros(1))[1])
    ws = None if have is None else torch.zeros(have, dtype=torch.uint8)
    lens = torch.tensor([5, 40, 70], dtype=torch.int32)
    pipeline.decode_layer(*[None] * 8, types.SimpleNamespace(page=16), torch.zeros(3, 9), lens, lens, positions=1, n_sel=3, bounds=1,
                          max_len=max_len, workspace=ws)
    assert asked == ([] if have is None else [(3, 2, max_len or 144)])
    assert got[0] is (ws if have is not None and have >= 100 else None) and got[1] is ws
