"""CPU-only: between them the tested products take every kernel of vsa2_int8_matmul, and the ranges of K fit the workspace."""
import random

import pytest

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild
from test_gpu_int8 import SHAPES


@pytest.fixture(scope="module", autouse=True)
def lib():
    vbuild.build_library()


def test_the_tested_products_take_every_kernel():
    kinds = {}
    for m, n, k in SHAPES:
        columns, pair, ranges, _, _ = vb.vsa2_debug_int8_matmul_plan(m, n, k)
        kinds.setdefault((columns, pair, ranges > 1), []).append(n % 8 == 0)
    assert set(kinds) == {(8, 1, False), (32, 1, False), (32, 1, True), (128, 1, False), (128, 1, True), (128, 2, False), (128, 2, True), (256, 2, False), (256, 2, True)}
    for kind, aligned in kinds.items():      # results that leave by tensor copies, and that do not
        assert kind[2] or kind[0] == 8 or (any(aligned) and not all(aligned)), kind


def test_no_product_takes_another_kernel():
    rng = random.Random(2)
    for _ in range(4000):
        m, n, k = (int(2 ** rng.uniform(0, e)) for e in (17, 15, 16.9))
        for pairs in (True, False):
            columns, pair, ranges, tiles, together = vb.vsa2_debug_int8_matmul_plan(m, n, k, pairs=pairs)
            assert (columns, pair) in ((8, 1), (32, 1), (128, 1), (128, 2), (256, 2)) and (pairs or pair == 1)
            assert 1 <= together <= max(tiles, 1) and 1 <= ranges <= 16
            if ranges > 1:      # [status][ranges of m rows of n, rounded up to four]
                assert 256 + 4 * ranges * m * (-(-n // 4) * 4) <= vb.vsa2_int8_matmul_workspace_bytes(m, n, k)
                assert ranges * tiles * -(-n // (128 * pair)) <= 148 // pair and ranges <= -(-k // 128)


def test_the_query_refuses_what_is_no_product():
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 1, 1)):
        with pytest.raises(vb.Vsa2Error):
            vb.vsa2_debug_int8_matmul_plan(*bad)
