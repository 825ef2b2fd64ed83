"""Which pages the layers of a ``DecodePath`` read and write: checks on the host."""
import gc

import pytest
import torch

import paper_2608_08097_amd as P
from paper_2608_08097_amd.path import DecodePath, LayerState

D = P.dims(1, 4, 2, 128, 16, 4)


def _pages():
    return [torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16) for _ in range(2)]


def _path():
    return DecodePath(D, 2, 2, *_pages(), torch.zeros(1, 4, dtype=torch.int32), streams=(None, None))


def _commit(path, st):
    rows = torch.zeros(1, 2, 2, 128, dtype=torch.bfloat16)
    n = [torch.zeros(1, dtype=torch.int32) for _ in range(3)]
    path.commit(st, rows, rows, torch.zeros(1, 2, dtype=torch.int32), *n)


def _passes_to_the_library(path, st):
    with pytest.raises(ValueError, match="must be a device tensor"):  # past the path's own checks
        _commit(path, st)


def _refused(path, st):
    with pytest.raises(RuntimeError, match="several layers on one tier"):
        _commit(path, st)


def test_layers_on_one_tier_are_not_committed():
    path = _path()
    a = path.new_layer()
    _passes_to_the_library(path, a)
    b = path.new_layer()
    _refused(path, a)
    _refused(path, b)
    del b
    gc.collect()
    _passes_to_the_library(path, a)
    other = LayerState(D, 2, 2, "cpu")  # a layer that the path did not make
    _refused(path, other)
    _refused(path, a)


def test_layers_on_pages_of_their_own_are_committed():
    path = _path()
    shared, own = path.new_layer(), _pages()
    layers = [path.new_layer(*_pages()), path.new_layer(*own)]
    for st in (shared, *layers):
        _passes_to_the_library(path, st)
    again = path.new_layer(*own)
    for st in (layers[1], again):
        _refused(path, st)
    _passes_to_the_library(path, layers[0])


def test_a_layer_s_pages():
    path = _path()
    k, v = _pages()
    lk, lv = _pages()
    table = torch.ones(1, 4, dtype=torch.int32)
    st, own, both = path.new_layer(), path.new_layer(k, v), path.new_layer(k, v, (lk, lv, table))
    path.set_local_source(lv, lk, table)
    same = lambda a, b: len(a) == len(b) and all(x is y for x, y in zip(a, b))  # noqa: E731
    assert same(path._tier(st), (path.host_k, path.host_v, path.block_table)) and same(path._local(st), (lv, lk, table))
    assert same(path._tier(own), (k, v, path.block_table)) and same(path._local(own), (k, v, path.block_table))
    assert same(path._tier(both), (k, v, path.block_table)) and same(path._local(both), (lk, lv, table))
    for bad in ((k,), (None, v), (None, None, (lk, lv, table))):
        with pytest.raises(ValueError, match="own pages"):
            path.new_layer(*bad)
