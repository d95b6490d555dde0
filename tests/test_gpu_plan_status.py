"""What a plan says when a request does not fit and another's pages are none."""
import numpy as np
import pytest

from packed_cases import pool_state
from paper_2403_08058_b200 import chai
from test_gpu_packed import check_plan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_tokens", [30, 9000])           # one launch, two
@pytest.mark.parametrize("order", [(0, 1, 2), (2, 1, 0), (1, 0, 2)])
def test_a_bad_page_comes_before_a_request_that_does_not_fit(n_tokens, order):
    page, max_pages = 8, 6
    seq, new = np.array([20, 47, 9])[list(order)], np.array([3, 30, 1])[list(order)]       # 47 + 30 is longer than a list
    bad, full = order.index(0), order.index(1)
    table, free, count = pool_state(seq, page, 60, max_pages, 1)
    assert check_plan(seq, new, table, free, count, n_tokens, page)["status"] == chai.CHAI_ERR_CACHE_FULL
    table[bad, 2] = -3                                      # the page that its next token goes to
    assert check_plan(seq, new, table, free, count, n_tokens, page)["status"] == chai.CHAI_ERR_BAD_PAGE
    new[full] = 0
    assert check_plan(seq, new, table, free, count, n_tokens, page)["status"] == chai.CHAI_ERR_BAD_PAGE


@pytest.mark.parametrize("n_tokens", [30, 9000])
def test_a_stack_entry_that_is_no_page_comes_before_a_request_that_does_not_fit(n_tokens):
    page, max_pages = 8, 6
    seq, new = np.array([16, 8, 0]), np.array([3, 100, 2])
    table, free, count = pool_state(seq, page, 60, max_pages, 2)
    free[count - 1] = 60
    assert check_plan(seq, new, table, free, count, n_tokens, page)["status"] == chai.CHAI_ERR_BAD_PAGE
