"""CPU-only: the products that the GPU tests run (fp8_shapes) take every kernel that a product can take on a B200, however the plan's constants are set."""
import math
import random

import pytest

from fp8_shapes import SHAPES
from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild

STORES = {"tensor copies": dict(c_aligned=True), "plain stores": dict(c_aligned=False), "fp32": dict(c_dtype=vb.F32)}


@pytest.fixture(scope="module", autouse=True)
def library():
    vbuild.build_library()


def variant(m, n, k, store, **kw):
    columns, ctas, swap, ranges, tiles, together = vb.vsa2_debug_fp8_matmul_plan(m, n, k, **STORES[store], **kw)
    return columns, ctas, bool(swap), ranges > 1, tiles > together, store


def test_tested_products_take_every_kernel():
    tested = {variant(m, n, k, store) for m, n, k in SHAPES for store in STORES if store != "tensor copies" or n % 8 == 0}
    rng = random.Random(1)
    log = lambda most: int(math.exp(rng.uniform(0.0, math.log(most))))
    for _ in range(100000):
        m, n, k = log(40000), log(20000), log(30000)
        for store in STORES:
            v = variant(m, n, k, store)
            # (groups of tiles are walked alike whether or not K is cut)
            assert v in tested or (v[3] and v[4] and (*v[:4], False, v[5]) in tested), (m, n, k, v)


def test_without_room_for_pairs_no_product_takes_one():
    for m, n, k in SHAPES:
        for store in STORES:
            for kw in (dict(pairs=False), dict(sms=1)):
                v = variant(m, n, k, store, **kw)
                assert v[0] in (32, 128) and v[1] == 1 and not v[2]


def test_ranges_fit_the_workspace_and_the_blocks():
    for m, n, k in SHAPES + [(1, 1, 1), (224, 37888, 300), (32, 18944, 8192), (128, 9472, 30000)]:
        for sms in (1, 2, 77, 132, 148, 200):
            columns, ctas, swap, ranges, tiles, _ = vb.vsa2_debug_fp8_matmul_plan(m, n, k, vb.F32, sms=sms)
            assert 1 <= ranges <= min(16, -(-k // 128))
            if ranges > 1:
                assert not swap and ranges * m * (-(-n // 4) * 4) * 4 + 256 <= vb.vsa2_fp8_matmul_workspace_bytes(m, n, k)


def test_refusals():
    for bad in ((0, 1, 1), (1, -1, 1), (1, 1, 0)):
        with pytest.raises(vb.Vsa2Error):
            vb.vsa2_debug_fp8_matmul_plan(*bad)
    with pytest.raises(vb.Vsa2Error):
        vb.vsa2_debug_fp8_matmul_plan(1, 1, 1, c_dtype=5)
