"""The rows that a 4-bit path ranks blocks from, where its caller does not say (CPU only)."""
import pytest
import torch

import paper_2608_08097_amd as P
from paper_2608_08097_amd.path_q4 import Q4Path


def _path(T, G, **kw):
    d = P.dims(2, 2 * G, 2, 128, 16, 8)
    return Q4Path(d, T, 3, 16, torch.zeros((2, 8), dtype=torch.int32), **kw)


@pytest.mark.parametrize("T,G,first,count", [(1, 4, 0, 1), (1, 64, 0, 1), (2, 4, 1, 1), (5, 4, 1, 4), (17, 4, 1, 16), (18, 4, 1, 16),
                                             (64, 4, 1, 16), (64, 1, 1, 63), (64, 5, 1, 12), (9, 8, 1, 8), (3, 33, 1, 1)])
def test_defaults_are_rows_that_the_scorer_takes(T, G, first, count):
    path = _path(T, G)
    assert (path.first_draft, path.num_draft) == (first, count)
    assert path.first_draft + path.num_draft <= T and path.num_draft * G <= 64


def test_given_rows_are_kept():
    path = _path(5, 4, first_draft=0, num_draft=2)
    assert (path.first_draft, path.num_draft) == (0, 2)
    path = _path(5, 4, first_draft=2)
    assert (path.first_draft, path.num_draft) == (2, 3)
    path = _path(64, 4, num_draft=20)  # more than the scorer takes: its refusal, not fewer rows
    assert (path.first_draft, path.num_draft) == (1, 20)
    path = _path(1, 4, first_draft=1, num_draft=0)
    assert (path.first_draft, path.num_draft) == (1, 0)
