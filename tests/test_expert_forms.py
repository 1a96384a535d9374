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


@pytest.mark.parametrize("case", [c for c in X.CASES if len(c[0]) * c[1] * c[2] * sum(c[0]) < 1e9], ids=str)
def test_a_lost_term_shows(case, monkeypatch):
    """What the whole numbers are for: without the last row of a run, the last value of a row, the last inner value, or h's second term, the plain form's results are others."""
    monkeypatch.setattr(X, "DEV", "cpu")
    b = X.Block(*case)
    (y, kept), (dx, dgu, dd, dw) = b.forward(X.few(case)), b.backward()
    last = case[3] + sum(case[0]) - 1
    e = max(e for e, c in enumerate(case[0]) if c)
    other = X.Block(*case)
    other.dy[last] = 0
    _, less_gu, less_d, _ = other.backward()
    assert (less_gu[e] != dgu[e]).any(1).any(1).all() and (less_d[e] != dd[e]).any()
    other = X.Block(*case)
    other.x[:, -1] = 0
    other.dy[:, -1] = 0
    assert (other.forward(X.few(case))[1][case[3]:last + 1] != kept[case[3]:last + 1]).any(0).any(1).all() and (other.backward()[3] != dw)[case[3]:last + 1].any()
    other = X.Block(*case)
    other.down[:, :, -1] = 0
    other.gate_up[:, 1, -1] = 0
    assert (other.forward(X.few(case))[0] != y)[case[3]:last + 1].any() and (other.backward()[0] != dx)[case[3]:last + 1].any()
    if X.few(case):
        assert (b.forward(False)[0] != y).any()
