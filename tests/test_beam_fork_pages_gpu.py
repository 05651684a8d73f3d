"""Page ids outside the pool in the tables of a fork: reported wherever a beam that counts holds one, and never followed."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from beam_helpers import fork
from test_beam_fork_gpu import Tables, _built      # noqa: F401  (_built: the fixture)

pytestmark = pytest.mark.gpu


class Owned:
    """owned[page]; a page outside the pool is not."""

    def __init__(self, flags):
        self.flags = flags

    def __getitem__(self, page):
        return bool(0 <= page < len(self.flags) and self.flags[page])


def _check(t, parent, status):
    op = t.call(parent)
    got = {k: v.cpu().numpy() for k, v in op.run().items()}
    torch.cuda.synchronize()
    assert t.dev.read_status() == status
    want = fork(parent, t.kv.reshape(-1), t.ids, t.base, Owned(t.owned), t.reserve.tolist(), t.used, t.P)
    assert want["status"] == 0
    ids, base = t.d["page_ids_out"].cpu().numpy(), t.d["pos_base_out"].cpu().numpy()
    for r, (p, b, n) in enumerate(want["rows"]):
        assert got["kv_len"][r] == n and ids[r, :len(p)].tolist() == p and base[r, :len(b)].tolist() == b
        assert (ids[r, len(p):] == -9).all() and (base[r, len(b):] == -9).all()
    c = want["copies"]
    assert got["n_copies"][0] == len(c) and got["reserve_used"][0] == want["used"]
    for name, i in (("copy_src", 0), ("copy_dst", 1), ("copy_slots", 2)):
        assert got[name].tolist() == [x[i] for x in c] + [-1] * (parent.size - len(c))
    assert t.d["reserve"].cpu().numpy().tolist() == want["reserve"]


@pytest.mark.parametrize("bad", [-1, "pool", 1 << 30, -(1 << 31)])
@pytest.mark.parametrize("W,context,grown", [(4, 30, 90), (7, 9003, 120)])
def test_where_a_beam_holds_a_page_that_is_none(W, context, grown, bad):
    t = Tables(16, G=2, W=W, P=16, context=context, grown=grown, ragged=False)
    assert (t.kv % 16 != 0).all()
    bad = t.num_pages if bad == "pool" else bad
    keep, last = t.ids.copy(), int(t.kv[0, 0]) // 16
    stay = np.tile(np.arange(W), (2, 1))
    drop = stay.copy()
    drop[0, 1] = 0                                                   # beam 1 of the first group is not continued
    for entry in (0, 1, last - 1, last, last + 1):
        for parent in (stay, drop, np.full((2, W), -1)):
            t.ids = keep.copy()
            t.ids[1, entry] = bad
            _check(t, parent, M.MEPIC_DEV_BAD_PAGE if entry <= last else 0)      # (an entry behind its length: nobody's)
    t.ids = keep.copy()
    t.ids[W:, 2] = bad                                               # the same for all beams of a group
    _check(t, stay, M.MEPIC_DEV_BAD_PAGE)
    t.ids = keep
    _check(t, drop, 0)
