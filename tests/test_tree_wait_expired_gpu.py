"""A bounded wait of the tree attention that runs out: status bit, a clean return, and parity right after."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200.build import build_library
from tree_helpers import TreeCase

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [128, 64])
def test_a_copy_that_never_comes(fp8, D):
    if fp8 and D != 128:
        pytest.skip("8-bit pages have head_dim 128")
    build_library()
    case = TreeCase(40, Hq=4, Hkv=1, D=D, P=16, specs=[(2000, 5), (60, 3)], fp8=fp8)
    case.device()
    batch = case.batch()
    for tile in (0, 1):
        M.mepic_kernel_test_hooks(spin_limit=20000, skip_tile=tile)      # tens of milliseconds, then the wait gives up
        try:
            batch.run(0.09)
            torch.cuda.synchronize()
        finally:
            M.mepic_kernel_test_hooks()
        assert case.dev.read_status() & M.MEPIC_DEV_WAIT_EXPIRED or tile >= 1      # CTA 0's piece may have one tile only
        case.dev.status.zero_()
        out = batch.run(0.09)
        torch.cuda.synchronize()
        assert case.dev.read_status() == 0
        case.check(out, 0.09)
