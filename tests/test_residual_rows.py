"""CPU-only: the rows that the CTAs of the norm forward take, also of matrices of more rows than a signed step of the walk would hold."""
import os
import re

import pytest

from paper_2609_32882_b200 import binding as vb
from paper_2609_32882_b200 import build as vbuild

MOST = 2 ** 31 - 1 - 2 ** 16      # rows that a call takes


@pytest.fixture(scope="module", autouse=True)
def lib():
    vbuild.build_library()


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 147, 148, 600, 4736, 18944, 18945, 18948, 75600, 1 << 30, 1717986916, 1717986917, 1717986920, 1750000000, MOST - 3, MOST])
@pytest.mark.parametrize("resident", [1, 148, 148 * 32])
def test_every_row_is_taken_once_and_none_behind_the_last(rows, resident):
    ctas = vb.vsa2_debug_residual_norm_rows(rows, resident, 0)[0]
    assert 1 <= ctas <= rows and ctas == (-(-rows // 4) if -(-rows // 4) > resident else min(rows, resident))
    for cta in sorted({0, 1 % ctas, ctas // 2, ctas - 2 if ctas > 1 else 0, ctas - 1}):
        of, taken, last = vb.vsa2_debug_residual_norm_rows(rows, resident, cta)
        assert of == ctas
        assert taken == -(-(rows - cta) // ctas)                      # rows cta, cta + ctas, .. below `rows`
        assert last == cta + (taken - 1) * ctas < rows


def test_the_query_refuses_what_is_no_launch():
    for bad in ((0, 148, 0), (MOST + 1, 148, 0), (10, 0, 0), (10, 148, -1), (10, 148, 10)):
        with pytest.raises(vb.Vsa2Error):
            vb.vsa2_debug_residual_norm_rows(*bad)


def test_walks_that_count_with_a_sign_have_a_grid_that_the_accepted_rows_leave_room_for():
    """A loop `for (int row = blockIdx.x; ..; row += gridDim.x)` forms numbers up to rows + CTAs: CTAs at most 2^16.  Only the backward has one (kNormParts CTAs)."""
    with open(os.path.join(vbuild.CSRC, "residual_norm.cu")) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    kernels = re.findall(r"\b(norm_\w+_kernel)\(const __grid_constant__[^{]*\{(.*?)\n\}", code, re.S)
    assert {name for name, _ in kernels} == {"norm_fwd_kernel", "norm_bwd_kernel"}
    for name, body in kernels:
        signed = re.search(r"for \(int row = blockIdx\.x;", body) is not None
        assert signed == (name == "norm_bwd_kernel") and signed != ("RowWalk walk{" in body)
    assert int(re.search(r"kNormParts = (\d+);", code).group(1)) <= 2 ** 16
    assert re.search(r"if \(ctas > kNormParts\) ctas = kNormParts;", code)
