"""Which kernel the router's rule takes, by the bits of its results."""
import pytest
import torch

import paper_2303_08999_amd as sr
from test_gpu_route import DEV, DT, PLANAR, PM, Guarded, logits, stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L", [8, 40, 72])
@pytest.mark.parametrize("zd", ["f32", "f16", "bf16"])
def test_few_rows_off_16_byte_pieces_go_where_planes_go(L, zd):
    """Rows of eight logits a load have a kernel of their own from the first pixel on; rows at an address that is not a multiple of 16 cannot be
    read so, and 1000 pixels of them are the wavefront kernel's, as planes are.  The two kernels sum in different orders: the same bits
    in every value are the same kernel's."""
    z = logits(1, L, 1, 1000, zd, 90 + L, special=False)
    T = min(L, 8)
    out = []
    for layout, shift in ((PLANAR, 0), (PM, 1)):
        coeff = Guarded(stored(z, layout, 1).shape, DT[zd], shift)
        coeff.t.copy_(stored(z, layout, 1))
        index, value = torch.empty((1, T, 1, 1000), device=DEV, dtype=torch.uint8), torch.empty((1, T, 1, 1000), device=DEV)
        sr.sr_list_route(coeff.t, L, 1, T, sr.SR_ROUTE_SOFTMAX, layout, None, index, value)
        out.append((index, value))
    torch.cuda.synchronize()
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
