"""The bounds that pd_paged_append_rope keeps are those of pd_paged_append to the bit, the signs of zeros among them."""

import pytest
import torch

from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16
from test_gpu_paged_rope import EPS, IDS, KINDS, Rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
@pytest.mark.parametrize("d", [64, 128])
def test_zeros_of_both_signs(gpu_lib, kind, d):
    """Channels that hold nothing but zeros: of one sign, of both in every order, beside larger and smaller elements; pages
    that begin with the call and pages that it widens."""
    R, n = 16, 64
    g = torch.Generator().manual_seed(4)
    rows = Rows(kind, [n], norm=False, rotate=False, new_len=n, hq=2, hkv=2, d=d, R=R, seed=6)
    x = rows.x[0]
    zeros = torch.where(torch.rand(n, 2, d, generator=g) < 0.5, 0.0, -0.0).to(x.dtype)
    zeros[:, :, 1], zeros[:, :, 2] = 0.0, -0.0
    zeros[:, :, 3] = zeros[:, :, 3].abs().neg() + 0.0
    zeros[::R, :, 4], zeros[R - 1::R, :, 5] = -0.0, 0.0
    zeros[5, :, 6], zeros[R + 5, :, 7] = 1.0, -1.0
    x[:, 2:4] = zeros
    bits = torch.int16 if kind[0] == PD_BF16 else torch.int32
    dims = _lib.PagedDims.from_buffer_copy(rows.case.dims)
    for cuts in ((0, n), (0, 1, 2, 3, n), (0, 7, 20, 33, n), tuple(range(n + 1))):
        held = []
        for rope in (False, True):
            c = rows.empty()
            for a, b in zip(cuts, cuts[1:]):
                dims.new_len = b - a
                y = x[None, a:b].cuda()
                c["kv_len"].fill_(b)
                c["new_rows"].fill_(b - a)
                if rope:
                    _lib.pd_paged_append_rope(dims, c["cache"], None, y[:, :, 2:4], y[:, :, 4:], None, None, EPS, None, 0.0, None)
                else:
                    _lib.pd_paged_append(dims, c["cache"], y[:, :, 2:4], y[:, :, 4:])
            held.append(c["bounds"].cpu()[rows.case.table[0].long()])
        assert torch.equal(held[0], held[1])
        off = held[0].view(bits) != held[1].view(bits)
        assert not off.any(), (cuts[:5], int(off.sum()), off.nonzero()[:5].tolist())
