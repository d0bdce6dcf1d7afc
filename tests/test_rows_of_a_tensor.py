"""What the binding makes of rows [..., heads, d]: pointer and row stride, for tensors of three and four dimensions."""

import itertools

import pytest
import torch

from paper_2606_10537_amd import _lib


def rows(t):
    return _lib._rows("t", t, tuple(t.shape), torch.float32, -1)


class NoStride(torch.Tensor):
    def stride(self, *a):
        raise AssertionError("a contiguous tensor's strides were asked for")


@pytest.mark.parametrize("shape", [(1, 3, 4), (5, 1, 4), (5, 3, 4), (3, 4)])
def test_contiguous_rows_are_told_first(shape):
    t = torch.zeros(shape).as_subclass(NoStride)
    assert rows(t) == (t.data_ptr(), shape[-2] * shape[-1])


def reference(t):
    """Row stride, or None: from the address of every element."""
    base, heads, d = t.data_ptr(), t.shape[-2], t.shape[-1]
    at = torch.tensor([t[i].data_ptr() - base for i in itertools.product(*map(range, t.shape))]).view(-1, heads, d) // 4
    if not torch.equal(at - at[:, :1, :1], (torch.arange(heads)[:, None] * d + torch.arange(d))[None].expand_as(at)):
        return None
    first = at[:, 0, 0]
    steps = (first[1:] - first[:-1]).unique()
    return heads * d if len(first) == 1 else int(steps[0]) if len(steps) == 1 else None


def test_every_layout():
    """Slices, transposes and expansions of all dimensions: the stride that the addresses have, or a refusal."""
    g = torch.Generator().manual_seed(1)
    pick = lambda lo, hi: int(torch.randint(lo, hi, (), generator=g))  # noqa: E731
    refused = 0
    for i in range(1500):
        dims = 3 + i % 2
        t = torch.zeros([pick(1, 5) for _ in range(dims - 1)] + [pick(1, 6)])
        for k in range(dims):
            lo = pick(0, t.shape[k])
            t = t.narrow(k, lo, pick(1, t.shape[k] - lo + 1)) if pick(0, 3) else t
            t = t[(slice(None),) * k + (slice(None, None, 2),)] if pick(0, 6) == 0 else t
        if pick(0, 5) == 0:
            t = t.transpose(pick(0, dims), pick(0, dims))
        if pick(0, 6) == 0:
            k = pick(0, dims)
            t = t.narrow(k, 0, 1).expand([3 if j == k else n for j, n in enumerate(t.shape)])
        want = reference(t)
        if want is None:
            refused += 1
            with pytest.raises(ValueError):
                rows(t)
        else:
            ptr, stride = rows(t)
            assert ptr == t.data_ptr() and (stride == want or t.numel() == t.shape[-1] * t.shape[-2]), (t.shape, t.stride())
    assert 100 < refused < 1000
