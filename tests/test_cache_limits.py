"""Limits of the shared-prefix attention that its arithmetic has (no GPU needed)."""
import ctypes
import math

import pytest

from paper_2609_36938_b200 import binding as B
from paper_2609_36938_b200 import build

UNSUPPORTED = 2


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.load()


def test_more_heads_than_segments_are_numbered_for(lib):
    """Quotients of the kernel's reciprocals are right below 2^20, and a grid has 65535 rows: so many heads, and no more."""
    at = ctypes.c_void_p(0x1000)      # never dereferenced: validation fails first

    def call(H, n):
        return lib.janus_attn_decode_shared(at, 1024, H, 128, at, 128 * n * 64, 128 * n, 128, ctypes.c_void_p(0x900000), 128 * n * 64, 128 * n, 128, n, 128, 64, 100, at, 1000, at, at, at, 3000, 0.1,
                                            at, None, at, 1 << 60, None, None)

    assert call(65536, 1) == UNSUPPORTED and call(1 << 20, 1 << 20) == UNSUPPORTED
    # 1024 sessions of a launch: segments of the prefix (whole chunks of up to 128 rows, two times as many as fill 128), of one session's own tokens
    for group in range(1, 65536):
        kv, rows, parts = 65535 // group, min(group, 128), -(-group // 128)
        assert -(-1024 * parts // (2 * (128 // rows))) * kv < 2 ** 20 and kv * parts < 2 ** 20, group


def test_quotients_by_reciprocals():
    """x / d as the kernel takes it: a product with the rounded reciprocal, one step either way.  For every quotient below 2^20 the product is off by less than one."""
    import numpy as np

    rng = np.random.default_rng(1)
    for d in [1, 2, 3, 6, 7, 14, 127, 128, 1000, 4102, 65535, 1 << 20, (1 << 30) - 1] + [int(math.exp(rng.uniform(0, math.log(2 ** 30)))) for _ in range(200)]:
        top = min(2 ** 30, d * 2 ** 20) - 1
        x = np.unique(np.concatenate([rng.integers(0, top + 1, 2000), np.array([0, top]), np.minimum(np.arange(1, 200) * d, top), np.minimum(np.arange(1, 200) * d - 1, top),
                                      top // d * d - np.arange(0, 2)])).astype(np.int64)
        x = x[x >= 0]
        inv = np.float32(1.0) / np.float32(d)
        q = np.floor(x.astype(np.float32) * inv).astype(np.int64)
        r = x - q * d
        q = q - (r < 0) + (r >= d)
        assert np.array_equal(q, x // d), d
