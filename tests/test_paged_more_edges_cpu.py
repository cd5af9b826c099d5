"""The paged cache's normed heads, appends, drafted trees and chosen pages at their edges, without a GPU."""
import numpy as np

from oracle import paged as O


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
