"""Requests that share pages end without giving them back: with a length of 0."""
import numpy as np
import pytest

from packed_cases import pool_state
from paper_2403_08058_b200 import chai
from test_gpu_packed import check_plan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_tokens", [40, 9000])
def test_shared_pages_stay_with_their_owner(n_tokens):
    page, max_pages, n_pages = 8, 6, 40
    table, free, count = pool_state([30, 0, 0, 17], page, n_pages, max_pages, 3)
    table[1, :3] = table[2, :3] = table[0, :3]              # 1 and 2 read 24 positions of 0
    want = check_plan(np.array([30, 0, 0, 17]), np.array([2, -1, -1, -1]), table, free, count, n_tokens, page)
    assert want["status"] == chai.CHAI_OK and int(want["free_count"][0]) == count + 3      # (the pages of request 3)
    stack = want["free_pages"][: count + 3].tolist()
    assert sorted(stack + want["block_table"][0, :4].tolist()) == list(range(n_pages))
    # the last one that has them ends with its length: they go back once
    after = check_plan(want["kv_lens"], np.array([-1, 0, 0, 0]), want["block_table"], want["free_pages"], count + 3, n_tokens, page)
    assert sorted(after["free_pages"].tolist()) == list(range(n_pages)) and int(after["free_count"][0]) == n_pages
