"""CPU-only: the product's workspace is what products up to its sizes can need, and no more than the ranges that they can be cut into."""
import random

import pytest

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild


@pytest.fixture(scope="module", autouse=True)
def library():
    vbuild.build_library()


def test_small_products_ask_for_little():
    bytes_of = vb.vsa2_fp8_matmul_workspace_bytes
    for m, n, k in ((1, 128, 128), (1000, 1000, 100), (75600, 15360, 128), (0, 5, 900), (5, 0, 900), (5, 5, 0)):
        assert bytes_of(m, n, k) == 256                       # (one block of K, or nothing: never cut)
    for m, n, k in ((1, 15360, 5120), (3, 5, 2048), (40, 260, 300), (300, 515, 1153)):
        assert bytes_of(m, n, k) <= 256 + min(16, -(-k // 128)) * m * (n + 3) * 4
    assert bytes_of(75600, 15360, 5120) == 256 + 148 * 128 * 224 * 4
    assert bytes_of(2 ** 30, 2 ** 30, 2 ** 30) == 256 + 148 * 128 * 224 * 4 and bytes_of(-1, 1, 1) == 0
    assert bytes_of(1, 2 ** 31 - 1, 2 ** 31 - 1) == 256 + 148 * 128 * 32 * 4


def test_one_workspace_serves_all_smaller_products():
    rng = random.Random(2)
    size = lambda: (rng.choice([1, 7, 32, 33, 128, 129, 300, 2000]), rng.choice([1, 100, 130, 700, 5000]), rng.choice([1, 129, 1000, 5000, 40000]))
    for _ in range(20000):
        m, n, k = size()
        part = rng.randint(1, m), rng.randint(1, n), rng.randint(1, k)
        room = vb.vsa2_fp8_matmul_workspace_bytes(m, n, k)
        assert vb.vsa2_fp8_matmul_workspace_bytes(*part) <= room
        ranges = vb.vsa2_debug_fp8_matmul_plan(*part, sms=rng.choice([1, 2, 33, 132, 148, 160]), pairs=rng.random() < 0.8)[3]
        if ranges > 1:
            assert 256 + ranges * part[0] * (-(-part[1] // 4) * 4) * 4 <= room
