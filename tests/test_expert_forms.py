"""The sizes of exact_experts.py reach every tile size of every product of the experts, whole tiles and tiles in parts, and both tile sizes of the matrices' gradients, by the rules
themselves: a rule that changes cannot leave kernels without a test.  No GPU needed."""
import os

import pytest

import exact_experts as X
import tile_rules

pytestmark = pytest.mark.skipif(not os.path.exists(tile_rules.HIPCC), reason="no hipcc")
TILES = [(form, parts) for form in (X.SMALL, X.MIDDLE, X.LARGE) for parts in (False, True)]


def _reached(found, product):
    return {(form, parts > 1) for products, _ in found for form, parts in (products[product],)}


def test_the_sizes_of_bf16_experts_reach_every_form():
    found = X.forms(X.CASES)
    for product in ("up", "down", "act", "dx"):
        assert _reached(found, product) >= set(TILES), product
    assert (X.FEW, False) in _reached(found, "up") and (X.FEW, False) in _reached(found, "down")
    assert {grads for _, grads in found} == {False, True}
    for case, (products, _) in zip(X.CASES, found):
        assert X.few(case) == (products["up"][0] == X.FEW) == (products["down"][0] == X.FEW), case


def test_the_sizes_of_experts_of_codes_reach_every_form():
    found = X.forms(X.CODE_CASES, unit=128)
    for product in ("up", "down"):
        assert _reached(found, product) >= set(TILES) | {(X.FEW, False)}, product


def test_the_sizes_of_products_of_codes_reach_every_form():
    got = tile_rules.values(("mw_few.h",), tuple("int8_form(%d, %d, %d, %d, false)" % (sum(c) + 3, len(c), n_out, n_in) for c, n_in, n_out in X.MATRIX_CASES))
    assert set(got) == {X.FEW, X.SMALL, X.MIDDLE, X.LARGE}


@pytest.mark.parametrize("n_rows,n,hidden,inter", [(1, 1, 8, 8), (640, 4, 7168, 2048), (16384, 4, 7168, 2048), (1 << 24, 3, 2048, 512), (160, 16, 4096, 1024), (161, 16, 4096, 1024)])
def test_both_products_have_few_rows_or_neither(n_rows, n, hidden, inter):
    first, second = tile_rules.values(("mw_few.h",), tuple("forward_forms(%d, %d, %d, %d).%s" % (n_rows, n, hidden, inter, k) for k in ("first", "second")))
    assert (first == X.FEW) == (second == X.FEW)
