"""Objects of a drafted-token step that go away, or are bound, in ways their users may choose."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library
from tree_helpers import TreeCase, dev32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"


@pytest.mark.parametrize("how", ["stream", "current stream"])
def test_memory_of_a_dropped_object_is_not_handed_out_while_its_kernels_run(how):
    case = TreeCase(80, Hq=8, Hkv=2, D=128, P=16, specs=[(300, 5), (40, 3)])
    case.device()
    side = torch.cuda.Stream()
    case.batch().run(0.09, side)                           # what happens once (kernels loaded, events made) is not waited for below
    torch.cuda.synchronize()
    batch = case.batch()
    size, at = batch.workspace.numel(), batch.workspace.data_ptr()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)                   # half a second: the call below is still in the queue when its object goes
    if how == "current stream":
        with torch.cuda.stream(side):
            out = batch.run(0.09)
    else:
        out = batch.run(0.09, side)
    del batch
    early = not side.query()                               # (asked first: a new allocation may itself wait for the GPU)
    other = torch.empty(size, dtype=torch.uint8, device="cuda:0")
    torch.cuda.synchronize()
    assert early, "the kernels were through before the memory was asked for"
    assert other.data_ptr() != at
    assert case.dev.read_status() == 0
    case.check(out, 0.09)


@pytest.mark.parametrize("how", ["raw handle", "ExternalStream", "current stream"])
def test_a_stream_of_the_callers_own_may_go_before_the_object(how):
    # the caller waits for the stream, destroys it and drops the object after: nothing may come back to the handle
    case = TreeCase(81, Hq=8, Hkv=2, D=128, P=16, specs=[(300, 5), (40, 3)])
    case.device()
    rt, handle = torch.cuda.cudart(), ctypes.c_ulonglong(0)
    assert int(rt.cudaStreamCreate(ctypes.addressof(handle))) == 0
    batch = case.batch()
    torch.cuda.synchronize()
    mine = torch.cuda.ExternalStream(handle.value, device=0)
    if how == "current stream":
        with torch.cuda.stream(mine):
            out = batch.run(0.09)
    else:
        out = batch.run(0.09, handle.value if how == "raw handle" else mine)
    mine.synchronize()
    assert int(rt.cudaStreamDestroy(handle.value)) == 0
    size = batch.workspace.numel()
    del batch
    other = torch.empty(size, dtype=torch.uint8, device="cuda:0")
    other.zero_()
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, 0.09)
