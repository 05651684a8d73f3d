"""A bounded wait of the tree attention that runs out while the pipeline is full: copies and products of other tiles are in
flight when the CTA gives up.  Status bit, a clean return, and parity right after, again and again."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200.build import build_library
from tree_helpers import TreeCase

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,fp8", [(128, False), (128, True), (64, False)])
@pytest.mark.parametrize("specs", [[(9000, 2), (9011, 1), (900, 3)],                               # a long run of tiles in one item
                                   [(int(100 + 37 * i % 500), 1 + i % 3) for i in range(48)]])     # items of a few tiles each
def test_a_copy_that_never_comes_in_a_full_pipeline(D, fp8, specs):
    build_library()
    case = TreeCase(41, Hq=8, Hkv=8, D=D, P=16, specs=specs, fp8=fp8)
    # CTA 0 takes the first piece of the one line there is: tiles / SMs, rounded down
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    tiles = int((-(-case.kv_len.astype(np.int64) // 128) + 1).sum()) * case.Hkv // sms
    assert tiles >= 6
    case.device()
    batch = case.batch()
    for tile in (0, 1, 3, 4, tiles - 1):
        M.mepic_kernel_test_hooks(spin_limit=20000, skip_tile=tile)      # tens of milliseconds, then the wait gives up
        try:
            batch.run(0.09)
            torch.cuda.synchronize()
        finally:
            M.mepic_kernel_test_hooks()
        assert case.dev.read_status() == M.MEPIC_DEV_WAIT_EXPIRED, tile
        case.dev.status.zero_()
        batch.out.zero_()
        out = batch.run(0.09)
        torch.cuda.synchronize()
        assert case.dev.read_status() == 0
        case.check(out, 0.09, which=[0, 2])
