"""Products of 8-bit rows (gf_block.h) in each form that the rule between the kernels leads to, against 64 bits.

Every case says which form it is there for and asserts that this form is what runs: a rule that is fitted anew may move the borders,
and then has to bring other sizes here.  Bounds as in test_fp8_gpu.py."""
import pytest
import torch

from block_util import DTYPES
from test_fp8_gpu import _check_product, _product

pytestmark = pytest.mark.gpu

F32, BF16 = DTYPES
WIDE, NARROW, BY_HAND = 1, 2, 4                 # many rows; tiles of 128 columns; results stored by the warps

# rows, N, K, gradient of the input, results, the form; the last tile lacks rows, and most lack columns
FORMS = [
    (4100, 1000, 576, False, BF16, WIDE),
    (4099, 1000, 576, False, F32, WIDE),
    (5000, 1000, 520, True, BF16, WIDE),
    (5001, 1000, 520, True, F32, WIDE),
    (18900, 96, 1000, False, BF16, WIDE | NARROW),
    (18900, 104, 1000, False, F32, WIDE | NARROW),
    (18000, 576, 96, True, BF16, WIDE | NARROW),               # the gradient through an expansion layer
    (18000, 576, 96, True, F32, WIDE | NARROW),
    (19001, 1000, 16, True, F32, WIDE | NARROW),               # fewer columns than a warp has
    (37000, 1000, 20, True, BF16, WIDE | NARROW | BY_HAND),
    (4099, 1001, 576, False, BF16, WIDE | BY_HAND),
    (4099, 1001, 576, False, F32, WIDE | BY_HAND),
    (4101, 1002, 576, False, BF16, WIDE | BY_HAND),            # rows 4 bytes further against the 16-byte places each time
    (4101, 1004, 576, False, BF16, WIDE | BY_HAND),            # and 8
    (5000, 1000, 513, True, BF16, WIDE | BY_HAND),
    (5000, 1000, 513, True, F32, WIDE | BY_HAND),
    (18900, 100, 1000, False, BF16, WIDE | NARROW | BY_HAND),
    (18901, 99, 1000, False, BF16, WIDE | NARROW | BY_HAND),
    (18900, 101, 1000, False, F32, WIDE | NARROW | BY_HAND),
    (18900, 1000, 100, True, BF16, WIDE | NARROW | BY_HAND),
    (18900, 1000, 101, True, F32, WIDE | NARROW | BY_HAND),
]


@pytest.mark.parametrize("M,N,K,transposed,out,form", FORMS, ids=lambda v: str(v).replace("torch.", ""))
def test_each_form_of_many_rows(gf, M, N, K, transposed, out, form):
    assert gf.gf_selftest_fp8_form(gf.make_fp8_matmul_desc(M, N, K, transposed=transposed, out_dtype=out)) == form
    _check_product(*_product(gf, M, N, K, transposed, out, (None, *DTYPES)[(M + N) % 3], seed=M + N + K), transposed)


@pytest.mark.parametrize("transposed", [False, True], ids=["layer", "input_gradient"])
@pytest.mark.parametrize("M", [9, 30, 150])
@pytest.mark.parametrize("chunks", [1, 2, 3, 4, 5, 6, 7, 8, 9, 13, 14, 17, 19, 25, 33])
def test_every_number_of_chunks_of_few_rows(gf, M, chunks, transposed):
    """Contractions of 128 terms and more, the last chunk a short one, dealt to the CTAs of a cluster evenly or not; results whole and not."""
    outer, inner = 260 + chunks % 2, 128 * chunks - 21
    N, K = (inner, outer) if transposed else (outer, inner)
    out = DTYPES[chunks % 2]
    assert not gf.gf_selftest_fp8_form(gf.make_fp8_matmul_desc(M, N, K, transposed=transposed, out_dtype=out)) & WIDE
    _check_product(*_product(gf, M, N, K, transposed, out, F32, seed=M + chunks), transposed)


def test_clusters_have_no_idle_cta(gf):
    """As many CTAs as there are shares of a half, quarter or eighth of the chunks, rounded up; not 3."""
    seen = set()
    for chunks in range(1, 200):
        for M, N in ((4, 640), (40, 640), (120, 640), (4, 10240)):       # (80 tiles: clusters of 2 at most)
            ctas = gf.gf_selftest_fp8_form(gf.make_fp8_matmul_desc(M, N, 128 * chunks, out_dtype=BF16)) >> 8
            if ctas:
                assert 1 <= ctas <= min(8, chunks) and ctas != 3
                seen.add(ctas)
    assert seen >= {1, 2, 4, 5, 6, 7, 8}
