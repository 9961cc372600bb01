"""The native marshalling holds the tensors that it gets from attributes until
its call has returned: a property may make them on the spot, and then nobody
else holds them. The library's entry points are replaced by functions that
look at the tensors, so nothing is launched on them."""
import ctypes
import weakref

import pytest
import torch

from paper_2607_29221_amd import mosaic as m
from tests.cache_util import clone, make_cache, same_bits, seeded

pytestmark = pytest.mark.gpu


class _Views:
    """Attributes of another object as views made on every access."""

    def __init__(self, of, refs):
        self.__dict__.update(of=of, refs=refs)

    def __getattr__(self, name):
        v = getattr(self.of, name)
        if isinstance(v, torch.Tensor):
            v = v.view(v.shape) if v.is_contiguous() else v[:]
            self.refs.append(weakref.ref(v))
        return v


@pytest.fixture
def bound():
    """The native functions with every entry point a function that notes how
    many of ``refs`` are alive."""
    b, refs, alive = m._native(), [], []

    def look():
        alive.append([r() is not None for r in refs])
        return 0
    stub = ctypes.CFUNCTYPE(ctypes.c_int32)(look)
    address = ctypes.cast(stub, ctypes.c_void_p).value
    real = tuple(ctypes.cast(getattr(m._lib.load(), n), ctypes.c_void_p).value for n in m._BOUND)
    rest = (torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, m._lib.MosaicRng)
    b.bind((address,) * len(real), *rest)
    yield b, refs, alive
    b.bind(real, *rest)


def _zeros(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def test_cache_and_rotary(bound):
    b, refs, alive = bound
    c = _Views(m.KVCache.empty(2, 40, 2, 64, page_size=16, evicts=True), refs)
    rotary = _Views(m.Rotary(m.Rotary.frequencies(8, 32), [16, 16], _zeros(2, 2)), refs)
    x, q = _zeros(2, 512, dtype=torch.float32), _zeros(2, 256, dtype=torch.float32)
    assert b.cache_append(c, x, 4, q, None, rotary, None) == 0
    assert len(refs) == 8 and alive == [[True] * 8]
    refs.clear(), alive.clear()
    assert b.cache_attend(c, x[:, :256], 4, q, None, None, True) == 0
    assert len(refs) == 6 and alive == [[True] * 6] * 2             # the workspace's size, then the call
    refs.clear(), alive.clear()
    assert b.cache_evict(c, 20, 2, None, None, None, None, None) == 0
    assert len(refs) == 6 and alive == [[True] * 6] * 2
    assert not any(r() is not None for r in refs)                   # and no longer


def test_digits_and_sparse_rows(bound):
    b, refs, alive = bound
    x, y = (_Views(m.Digits.empty(rows, 64), refs) for rows in (2, 3))
    assert b.masked_matmul(x, y, 2, 3, 64, _zeros(2, 3)) == 0
    assert len(refs) == 2 and alive == [[True, True]]
    refs.clear(), alive.clear()
    p = _Views(m.SparseRows(_zeros(4, dtype=torch.int64), _zeros(4), _zeros(4), 3, 64), refs)
    assert b.cols_terms([(p, _zeros(8, 64)), (p, _zeros(8, 64))], 8, _zeros(8, 3), False, None, None, None, None) == 0
    assert len(refs) == 6 and alive and all(a == [True] * 6 for a in alive)
    assert not any(r() is not None for r in refs)


def test_views_give_what_plain_tensors_give():
    c = make_cache((30, 45), 2, 64, 16, "bf16", 5, room=4, evicts=True)
    other = clone(c)
    x = torch.randn((2, 512), generator=seeded(6), device="cuda")
    got = []
    for cache in (c, _Views(other, [])):
        q, out = torch.empty((2, 256), device="cuda"), torch.empty((2, 256), device="cuda")
        b = m._native()
        assert b.cache_append(cache, x, 4, q, None, None, None) == 0
        assert b.cache_attend(cache, q, 4, out, None, None, True) == 0
        assert b.cache_evict(cache, 25, 2, None, None, None, None, None) == 0
        got.append((q, out))
    assert all(torch.equal(*p) for p in zip(*got))
    assert same_bits(c.k, other.k) and same_bits(c.weights, other.weights) and torch.equal(c.state, other.state)
