"""Arrays that rotary positions make and refuse, without a kernel."""
import pytest
import torch

from paper_2403_08058_b200 import chai


def rows_of(x):
    """Storage offsets of all elements."""
    offsets = torch.zeros(x.shape, dtype=torch.int64)
    for d, (n, s) in enumerate(zip(x.shape, x.stride())):
        offsets += (torch.arange(n) * s).view([-1 if i == d else 1 for i in range(4)])
    return offsets.flatten()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,H,N,D", [(1, 1, 1, 64), (2, 3, 5, 64), (1, 4, 1, 128), (3, 1, 7, 64), (2, 1, 1, 64)])
def test_new_arrays_are_dense(B, H, N, D, dtype):
    z = lambda *shape: torch.zeros(*shape, dtype=dtype)
    fused = z(B, N, 3, H, D)
    arrays = {
        "dense": z(B, H, N, D), "tokens first": z(B, N, H, D).transpose(1, 2), "heads first": z(H, B, N, D).transpose(0, 1),
        "requests last": z(H, N, B, D).permute(2, 0, 1, 3),
        "part": fused[:, :, 1].transpose(1, 2), "slice": z(B, H + 2, N + 3, D)[:, 1:-1, 2:-1], "every second": z(2 * B, H, 2 * N, D)[::2, :, ::2],
        "shared": z(1, H, 1, D).expand(B, H, N, D), "shared heads": z(B, 1, N, D).expand(B, H, N, D),
        "windows": z(B, H, (N - 1) * 16 + D).unfold(2, D, 16), "overlapping heads": z(B * 4096).as_strided((B, H, N, D), (4096, 16, 256, 1)),
    }
    for name, x in arrays.items():
        y = chai._rotated_like(x)
        assert y.shape == x.shape and y.dtype is x.dtype and y.stride(3) == 1, name
        assert sorted(rows_of(y).tolist()) == list(range(x.numel())), name        # every element once, no gap
        assert y.untyped_storage().nbytes() == x.numel() * x.element_size(), name
    for name in ("dense", "tokens first", "heads first", "requests last"):
        assert torch.equal(rows_of(chai._rotated_like(arrays[name])), rows_of(arrays[name])), name
    assert chai._rotated_like(arrays["part"]).transpose(1, 2).is_contiguous()


# ---- refusals: addresses are numbers here, for what is refused is never read, and without a device nothing else is ----

D, F32, AT = 64, 0, 1 << 40


def rope(q, k, q_out, k_out, B, Hq, Hk, N, strides):
    """Addresses in elements of fp32; strides: of q, q_out, k, k_out.  The status, and the refusal's text."""
    import ctypes
    lib = chai.load()
    at = lambda x: None if x is None else AT + 4 * x
    flat = (ctypes.c_int64 * 12)(*[s for array in strides for s in array])
    rc = lib.chai_rope(at(q), at(k), at(q_out), at(k_out), None, AT, B, Hq, Hk, N, D, 64, 0, None, flat, F32, None)
    return rc, lib.chai_last_error().decode()


def places(base, strides, sizes):
    return {base + b * strides[0] + h * strides[1] + n * strides[2] for b in range(sizes[0]) for h in range(sizes[1]) for n in range(sizes[2])}


def meet(x, y):
    y = sorted(y)
    import bisect
    for p in x:
        i = bisect.bisect(y, p - D)
        if i < len(y) and y[i] < p + D:
            return True
    return False


REFUSED = chai.CHAI_ERR_INVALID_ARG


def test_refused_overlaps():
    dense, far = (2 * 3 * D, 3 * D, D), 1 << 20
    zero = (0, 0, 0)
    go = lambda q, q_out, s=dense, s_out=dense, **kw: rope(q, None, q_out, None, 2, 2, 0, 3, (s, s_out, zero, zero))
    for shift in (4, D - 4, D, 5 * D, 11 * D, 11 * D + D - 4):                   # a row further or many
        for sign in (1, -1):
            rc, text = go(far, far + sign * shift)
            assert rc == REFUSED and "overlap an input" in text, shift
    rc, text = go(far, far, (2 * 3 * D, D, 2 * D))                               # the same array, other strides
    assert rc == REFUSED and "overlap an input" in text
    rc, text = go(far, far, (0, 3 * D, D))                                       # one request's rows for both
    assert rc == REFUSED and "overlap an input" in text
    for s in ((6 * D, 3 * D, D - 4), (6 * D, 2 * D, D), (5 * D, 3 * D, D), (D, 3 * D, D), (6 * D, 3 * D, 3 * D + 4)):
        rc, text = go(0, far, dense, s)
        assert rc == REFUSED and "rows of an output" in text, s
    two = lambda q_out, k_out, q=0, k=8 * far: rope(q, k, q_out, k_out, 2, 2, 2, 3, (dense,) * 4)
    for shift in (0, 4, 11 * D, -11 * D):
        rc, text = two(4 * far, 4 * far + shift)
        assert rc == REFUSED and "outputs must not" in text, shift
    for q_out, k_out in ((8 * far, far), (8 * far + 4, far), (far, 0), (far, D)):     # onto the other's input
        rc, text = two(q_out, k_out)
        assert rc == REFUSED and "overlap an input" in text, (q_out, k_out)


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused would run on addresses that are none")
def test_refused_are_the_ones_that_overlap():
    import random
    rng = random.Random(7)
    seen = [0, 0]
    for _ in range(4000):
        sizes = [rng.choice((1, 2, 3, 4)) for _ in range(3)]
        order = rng.sample(range(3), 3)
        strides, span = [0] * 3, D
        for i in order:                                                           # nested, with room between
            strides[i] = (span + rng.choice((0, 0, 4, D, 3 * D, 200)) + 3) // 4 * 4
            span += (sizes[i] - 1) * strides[i]
        strides = tuple(strides)
        base, to = 1 << 20, (1 << 20) + rng.randint(-span // 4 - 8, span // 4 + 8) * 4
        zero = (0, 0, 0)
        want = to != base and meet(places(base, strides, sizes), places(to, strides, sizes))
        rc, text = rope(base, None, to, None, sizes[0], sizes[1], 0, sizes[2], (strides, strides, zero, zero))
        assert (rc == REFUSED and "overlap" in text) == want, (sizes, strides, to - base)
        # the same arrays as two outputs, of different numbers of heads
        heads = rng.choice((1, sizes[1]))
        far = 1 << 28
        want_two = meet(places(base, strides, sizes), places(to, strides, [sizes[0], heads, sizes[2]]))
        rc, text = rope(far, 2 * far, base, to, sizes[0], sizes[1], heads, sizes[2], (strides,) * 4)
        assert (rc == REFUSED and "outputs" in text) == want_two, (sizes, heads, strides, to - base)
        seen[want_two] += 1
    assert min(seen) > 500
