"""The index arithmetic of reading back, of windows and of the shared prefix's partial sums, compiled for the host from the header that the kernels include: ragged batches,
empty sequences, tables too narrow, arrays full of garbage."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import streaming_oracle as o

HERE = os.path.dirname(os.path.abspath(__file__))


def test_places_of_views(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    exe = str(tmp_path / "views")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall",
                        os.path.join(HERE, "stream_views_check.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout, r.stderr[-2000:])


def _small(seed=0):
    rng = np.random.RandomState(seed)
    k, v = rng.randint(0, 0x60, (9, 2, 32, 64)).astype(np.uint8), rng.randint(0, 0x60, (9, 2, 64, 32)).astype(np.uint8)
    s = np.full((9, 2), 2.0 ** -5, np.float32)
    return k, v, s, s, rng.randn(12, 4, 64)


def test_a_window_without_an_end_is_all_of_the_cache():
    k, v, ks, vs, q = _small()
    cu, lens, table = np.array([0, 7, 12]), np.array([90, 60]), np.array([[0, 1, 2], [5, 3, -1]])
    want = o.attend(q, k, v, ks, vs, cu, lens, table, True)
    got = o.attend_window(q, k, v, ks, vs, cu, lens, table, 1, 1000, 0)
    assert np.allclose(got[0], want[0], atol=1e-12) and np.allclose(got[1], want[1], atol=1e-12)
    # sinks that reach as far make the window irrelevant
    got = o.attend_window(q, k, v, ks, vs, cu, lens, table, 1, 1, 1000)
    assert np.allclose(got[0], want[0], atol=1e-12)
    # a window of one token is that token's value
    o1, _ = o.attend_window(q, k, v, ks, vs, cu, lens, table, 1, 1, 0)
    assert np.allclose(o1[0, 0], o.decode(v[table[0, 83 // 32], 0, :, 83 % 32]) * 2.0 ** -5)


def test_a_prefix_is_the_sequence_in_front():
    """Pages of a prefix in front of a sequence's own pages, as one sequence, where the prefix ends with a page."""
    k, v, ks, vs, q = _small(1)
    cu, lens, table = np.array([0, 5, 12]), np.array([40, 9]), np.array([[4, 5], [6, 7]])
    prefix = (np.array([0, 12]), np.array([64]), np.array([[2, 8]]))
    want = o.attend(q, k, v, ks, vs, cu, lens + 64, np.array([[2, 8, 4, 5], [2, 8, 6, 7]]), True)
    got = o.attend_shared(q, k, v, ks, vs, prefix, (cu, lens, table), True)
    assert np.allclose(got[0], want[0], atol=1e-12) and np.allclose(got[1], want[1], atol=1e-12)


def test_reading_back_by_hand():
    k, v, ks, vs, _ = _small(2)
    K, V = o.read(k, v, ks, vs, np.array([1, 3]), np.array([33]), np.array([[3, 6]]), 4)
    assert (K[0] == -1e300).all() and (K[3] == -1e300).all()
    assert np.array_equal(K[1], o.decode(k[3, :, 31]) / 32) and np.array_equal(V[2], o.decode(v[6, :, :, 0]) / 32)
