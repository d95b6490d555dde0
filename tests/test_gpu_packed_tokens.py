"""One row for many tokens is refused by the packed calls; a copy of it is taken."""
import pytest
import torch

from packed_cases import DEV, i32, attend, batch, check, pages_of
from paper_2403_08058_b200 import chai

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache,io", [("bf16", "bf16"), ("e4m3", "f32")])
def test_rows_that_tokens_share(cache, io):
    n = 7
    c = batch(cache, io, 4, 2, 64, 16, [40], [n], seed=3)
    shared = c["q"][:1].clone().expand(n, -1, -1)
    own = shared.contiguous()
    c["q"] = shared
    with pytest.raises(ValueError, match="rows of its own"):
        attend(c)
    c["q"] = own
    check(c, attend(c))
    fn = chai.chai_append_rope_paged_fp8 if cache == "e4m3" else chai.chai_append_rope_paged
    turns, m = chai.chai_rope_frequencies(64, device=DEV)
    where = (c["reps"], i32([0] * n), i32(list(range(n))), c["table"][0, 0].long() * 16 + torch.arange(n, device=DEV), turns, m)
    for i in range(3):
        qkv = [own, own, own]
        qkv[i] = shared
        with pytest.raises(ValueError, match="qkv"[i] + " must have rows of its own"):
            fn(*qkv, *pages_of(c), *where)
    q = fn(own, own, own, *pages_of(c), *where)
    one = fn(own[:1], shared[:1], own[:1], *pages_of(c), c["reps"], i32([0]), i32([0]), where[3][:1], turns, m)
    assert torch.equal(one[0], q[0])
