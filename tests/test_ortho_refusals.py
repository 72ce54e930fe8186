"""What the orthogonalisation refuses of sizes and coefficients: calls with arguments that are no arrays (nothing is launched)."""
import os

import pytest

N, S, P, D, W, OK = -1, -2, -3, -4, -5, 0


@pytest.fixture(scope="module")
def call():
    from paper_2506_15050_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    lib = binding.load()

    def call(rows=100, cols=70, steps=5, a=3.4, b=-4.8, c=2.0, ws_bytes=0):
        return lib.tppo_orthogonalize(256, 1, rows, cols, cols, 0, 0, steps, a, b, c, 1e-7, 1.0, 256, cols, 0, 256, ws_bytes, None)
    return call


def test_iterations_that_shrink(call):
    """a^(steps - 1) below 2^-12; what is not refused for that has no workspace."""
    assert call(steps=14, a=0.5) == P and call(steps=14, a=-0.5) == P and call(steps=24, a=0.6) == P
    assert call(steps=2, a=0.0) == P and call(steps=2, a=0.0002) == P
    assert call(steps=13, a=0.5) == W and call(steps=2, a=0.00025) == W and call(steps=64, a=0.9) == W
    assert call(steps=1, a=0.0) == W and call(steps=0, a=0.0) == W and call(steps=64, a=1.0) == W


def test_sides(call):
    """A vocabulary of 152064 is a side like any other; beyond 262144, or 2^32 entries, none is."""
    assert call(rows=152064, cols=5120) == W and call(rows=5120, cols=152064) == W and call(rows=262144, cols=16384) == W
    assert call(rows=262145) == S and call(cols=262145) == S and call(rows=262144, cols=16385) == S and call(rows=65537, cols=65536) == S
    assert call(rows=1 << 40, cols=1 << 40) == S
