"""Group norm and 8-bit checkpoints at the ends of their range, against 64-bit references. Tolerances are derived at the tests."""
import numpy as np
import pytest
import torch

import oracle
from paper_1901_09290_b200 import binding as B
from paper_1901_09290_b200 import workloads as W
from tests import helpers as Hh

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ checkpoints
@pytest.mark.parametrize("npix,ldq", [(257, (1 << 24) + (1 << 17)), (5, (1 << 31) - 8)])
def test_codes_of_a_pitch_that_passes_32_bits_within_a_block(npix, ldq):
    """Pixels whose codes lie 4 GB apart while one thread block covers them all: each is where its pitch says, and nothing else is written."""
    c, C = Hh.ctx(), 8
    gen = torch.Generator().manual_seed(21)
    x = W.bf16_round(torch.randn((npix, C), generator=gen)).bfloat16().cuda()
    dense, scales = B.checkpoint_buffers(npix, C)
    B.pt_act_pack(c, B.make_pack_desc(npix, C), x, dense, scales)
    wide = torch.zeros((npix, ldq), dtype=torch.int8, device="cuda")
    d, wide_scales, back = B.make_pack_desc(npix, C, C, ldq), torch.zeros_like(scales), torch.zeros_like(x)
    B.pt_act_pack(c, d, x, wide, wide_scales)
    B.pt_act_unpack(c, d, wide, wide_scales, back)
    torch.cuda.synchronize()
    c.poll()
    assert torch.equal(wide[:, :C], dense) and torch.equal(wide_scales[:npix], scales[:npix])
    assert int(torch.count_nonzero(wide)) == int(torch.count_nonzero(dense))
    want = oracle.act_unpack(dense.cpu().numpy(), scales[:npix].cpu().numpy().reshape(npix, 1))
    assert np.array_equal(back.float().cpu().numpy().astype(np.float64), want)
