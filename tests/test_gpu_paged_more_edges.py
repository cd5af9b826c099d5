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
