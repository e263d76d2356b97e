"""Calls of the residual-block operators (include/gf_block.h) at the ends of what they take, as far as the host decides."""


def test_which_product_kernel(gf):
    """Nothing is said of a descriptor that is refused, or of no rows; few rows are few at any size."""
    f, mk = gf.gf_selftest_fp8_form, gf.make_fp8_matmul_desc
    assert gf.lib().gf_selftest_fp8_form(None) == -1
    for bad in ({"M": -1}, {"M": 0}, {"N": 0}, {"K": 0}, {"transposed": 2}, {"out_dtype": 3}, {"K": (1 << 24) + 1}):
        assert f(mk(**({"M": 4, "N": 8, "K": 8} | bad))) == -1
    for t in (False, True):
        for M in (1, 16, 17, 32):
            form = f(mk(M, 4096, 4096, transposed=t))
            assert form & 255 == 0 and 1 <= form >> 8 <= 8
