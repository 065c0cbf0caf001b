"""The plain definitions that the cache operators are tested against, pinned by cases worked out by hand and by invariants;
and what the library refuses without a device."""
import ctypes
import math

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2511_12280_b200 import binding as B_
from paper_2511_12280_b200 import build as build_mod


def test_rope_by_hand():
    # theta 100, two pairs, position 3: the first pair turns by 3, the second by 3 / 10
    a = co.rope_angles(np.array([[3]]), [2], 100.0, False)
    assert np.allclose(a, [[3.0, 0.3]], atol=1e-15)
    x = np.array([[[1.0, 0.0, 0.0, 2.0]]])
    assert np.allclose(co.rope(x, a), [[[math.cos(3), -2 * math.sin(0.3), math.sin(3), 2 * math.cos(0.3)]]])
    assert np.allclose(co.rope(x, a, neighbours=True), [[[math.cos(3), math.sin(3), -2 * math.sin(0.3), 2 * math.cos(0.3)]]])


def test_rope_axes_and_ladders():
    pos = np.array([[5, 7, 11]])
    shared = co.rope_angles(pos, [1, 2, 1], 16.0, False)
    assert np.allclose(shared, [[5.0, 7.0 / 2, 7.0 / 4, 11.0 / 8]])
    own = co.rope_angles(pos, [1, 2, 1], 16.0, True) % (2 * math.pi)
    assert np.allclose(own, np.array([[5.0, 7.0, 7.0 / 4, 11.0]]) % (2 * math.pi))


def test_rope_scores_depend_on_distance_alone_and_inverse_undoes():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    at = lambda p: co.rope_angles(np.array([[p, p]]), [3, 5], 1e4, True)
    dot = lambda x, y: float((x * y).sum())
    d = [dot(co.rope(q, at(p + 9)), co.rope(k, at(p))) for p in (0, 4, 1000003)]
    assert np.allclose(d, d[0], atol=1e-9)
    assert np.allclose(co.rope(co.rope(q, at(77)), at(77), inverse=True), q, atol=1e-12)


def test_attend_by_hand():
    q = np.array([[[1.0, 0.0], [0.0, 0.0]]])                        # one row, two heads sharing one key head
    k, v = np.array([[[math.log(3.0), 5.0]], [[0.0, -1.0]]]), np.array([[[4.0, 0.0]], [[0.0, 8.0]]])
    out, p, _, _ = co.attend(q, k, v, 1.0)
    assert np.allclose(p, [[[0.75, 0.25], [0.5, 0.5]]]) and np.allclose(out, [[[3.0, 2.0], [2.0, 4.0]]])
    out, p, _, _ = co.attend(q, k[:0], v[:0], 1.0)
    assert not out.any() and p.shape == (1, 2, 0)


def test_evict_by_hand():
    w = [3.0, 1.0, 2.0, 5.0, 1.0, 4.0]
    # kept: 5.0, 4.0, 3.0 at slots 3, 5, 0; the gaps 1 and 2 are filled in order
    assert co.evict(w, None, 3) == (3, [(3, 1), (5, 2)])
    assert co.evict(w, None, 5) == (5, [(5, 4)])                    # of the two lightest the later one goes
    assert co.evict(w, range(6), 3, protect_from=4) == (3, [(3, 0), (4, 1), (5, 2)])
    assert co.evict([0.0, math.nan, math.inf, -math.inf], None, 2) == (2, [(2, 0)])
    assert co.evict([-0.0, 0.0], None, 1) == (1, [])
    assert co.evict(w, None, -2) == (0, []) and co.evict(w, None, 9) == (6, []) and co.evict([], None, 3) == (0, [])


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B_.load()


def test_no_context_is_refused(lib):
    spec, cache = B_.RopeSpec([8]), B_._CacheStruct()
    assert lib.d3tom_rope(None, 0, ctypes.byref(spec), None, None, None, 1, 1, 0, None, None, None) == B_.ERR_INVALID_ARG
    assert lib.d3tom_cache_append(None, 0, ctypes.byref(cache), None, None, None, None, None, None, None, None, 1, 1, None,
                                  None) == B_.ERR_INVALID_ARG
    assert lib.d3tom_attn_cached(None, 0, ctypes.byref(cache), None, None, 1, 1, 1, 1, 1.0, 0, None, None, None) == B_.ERR_INVALID_ARG
    assert lib.d3tom_cache_evict(None, 0, ctypes.byref(cache), None, None, 1, 1, None, None) == B_.ERR_INVALID_ARG


def test_rope_spec_of_other_than_one_to_three_axes_is_refused():
    for bad in ([], [1, 2, 3, 4]):
        with pytest.raises(ValueError):
            B_.RopeSpec(bad)
