"""Selection over beams and vocabulary (mepic_beam_select) against its definition in 64 bits.

A score's error: the sum of exponentials has terms off by 2^-21 at most (ex2.approx 2^-22.5, the argument's rounding 2^-24 of
at most 8 for terms that matter) and at most 64 of them are added up in fp32 (64 x 2^-24): 5e-6 in the logarithm, and one rounding
of the score to fp32, 2^-24 of it.  Candidates further apart than 2e-5 (or exactly equal ones) have to come in order."""
import numpy as np
import pytest
import torch

import paper_2512_16822_b200 as M
from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library
from beam_helpers import select_group, dev32

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
CFG = M.Config(16, 8, 2, 128, 4, 64, 1e4)


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"


def _check(logits, scores, done, K, eos, pad, got, status):
    G, W = scores.shape
    x = logits.double().cpu().numpy().reshape(G, W, -1)
    got = {k: v.cpu().numpy() for k, v in got.items()}
    bad = False
    for g in range(G):
        want, b = select_group(x[g], scores[g], None if done is None else done[g], K, eos, pad)
        bad = bad or b
        n = min(len(want), K)
        for k in range(K):
            have = (int(got["parent"][g, k]), int(got["token"][g, k]), int(got["done"][g, k]))
            if k >= n:
                assert have == (-1, -1, 0) and got["score"][g, k] == -np.inf and got["n_new"][g, k] == 0, (g, k, have)
                continue
            s = want[k][0]
            gaps = [abs(s - want[i][0]) for i in (k - 1, k + 1) if 0 <= i < len(want)]
            if all(d == 0 or d > 2e-5 for d in gaps):
                assert have == want[k][1:], (g, k, have, want[k])
            assert abs(float(got["score"][g, k]) - s) <= 5e-6 + abs(s) * 2.0 ** -24, (g, k)
            assert got["n_new"][g, k] == 1 - have[2]
        assert len({(int(p), int(t)) for p, t in zip(got["parent"][g, :n], got["token"][g, :n])}) == n
    assert status == (M.MEPIC_DEV_BAD_LOGITS if bad else 0)


def _run(logits, scores, done=None, K=None, eos=None, pad=0):
    dev = RT.Device(CFG)
    op = RT.BeamSelect(dev, logits=logits, scores=torch.from_numpy(np.asarray(scores, dtype=np.float32)).cuda(),
                       done=None if done is None else dev32(done), n_select=K, eos_token=eos, pad_token=pad)
    op.workspace.fill_(255)
    got = op.run()
    torch.cuda.synchronize()
    _check(logits, np.asarray(scores, dtype=np.float32).astype(np.float64), done, scores.shape[1] if K is None else K, -1 if eos is None else eos, pad,
           got, dev.read_status())
    return op, dev


def _op(logits, scores, K):
    dev = RT.Device(CFG)
    return RT.BeamSelect(dev, logits=logits, scores=torch.from_numpy(np.asarray(scores, dtype=np.float32)).cuda(), n_select=K), dev


def _logits(rows, V, dtype, seed, std=2.5):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return (torch.randn((rows, V), generator=g, device="cuda:0") * std).to(TYPES[dtype])


def _scores(G, W, seed):
    return -np.random.default_rng(seed).uniform(0, 6, size=(G, W))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 33, 255, 2048, 8191, 8192, 8193, 16384, 16385, 40001])
def test_vocabularies_at_the_edges_of_pieces_and_segments(dtype, V):
    _run(_logits(6, V, dtype, V), _scores(2, 3, V), K=4, eos=V // 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("off", [0, 1, 3, 5])
def test_rows_of_any_alignment(dtype, off):
    # rows 1,003 + 5 elements apart, the first `off` elements into the buffer: each begins somewhere else in its 16 bytes; what
    # lies around them would win
    buf = torch.full((8, 1003 + 5), 3e4, device="cuda:0").to(TYPES[dtype])
    x = buf.view(-1)[off:off + 7 * 1008 + 1003].as_strided((8, 1003), (1008, 1))
    x.copy_(_logits(8, 1003, dtype, off))
    _run(x, _scores(2, 4, off), K=8)


@pytest.mark.parametrize("G,W,K", [(1, 1, 1), (1, 1, 64), (3, 32, 64), (5, 32, 1), (2, 8, 16), (70, 2, 3), (1, 17, 33)])
@pytest.mark.parametrize("V", [100, 20011])
def test_widths_and_numbers_of_candidates(G, W, K, V):
    _run(_logits(G * W, V, "fp32", G + W), _scores(G, W, K), K=K, eos=3)


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_logits_come_in_order_of_beam_and_token(dtype):
    x = torch.zeros((6, 30000), device="cuda:0", dtype=TYPES[dtype])
    op, _ = _run(x, np.zeros((2, 3)), K=40)                       # every candidate of every beam is equal
    assert op.parent[0].tolist() == [0] * 40 and op.token[0].tolist() == list(range(40))
    x[:, 20000:] = 1.0                                              # the best lie in a later segment, -0 and 0 are one value
    x[:, ::2] *= -1.0
    x[:, 25000:] = torch.where(x[:, 25000:] == -1, torch.ones_like(x[:, 25000:]), x[:, 25000:])
    _run(x, np.zeros((2, 3)), K=40)
    x = torch.round(_logits(6, 30000, "fp32", 1, 1.0)).to(TYPES[dtype])      # a few values only
    _run(x, np.array([[0.0, 0.0, -1.0], [0.0, -0.5, 0.0]]), K=64)
    row = _logits(1, 30000, dtype, 2)
    _run(row.expand(6, 30000).contiguous(), np.zeros((2, 3)), K=9)  # three beams with the same logits and the same score


@pytest.mark.parametrize("dtype", TYPES)
def test_sorted_rows(dtype):
    # all of the best in one stretch of neighbours, at either end
    x = torch.linspace(-20, 20, 50000, device="cuda:0").to(TYPES[dtype]).expand(2, 50000).contiguous()
    _run(x, _scores(1, 2, 5), K=64)
    _run(x.flip(1).contiguous(), _scores(1, 2, 5), K=64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("every,of", [(4, 16), (1, 16), (2, 5)])
def test_the_best_in_a_few_stretches_of_a_large_vocabulary(dtype, every, of):
    # whole stretches of 8,192 or 16,384 tokens stand above the rest of all rows: hundreds of neighbours are candidates
    V = 120000
    x = _logits(8, V, dtype, 15)
    stretch = 8192 if dtype == "fp32" else 16384
    lift = (torch.arange(V, device="cuda:0") // stretch)[None, :] + -(-V // stretch) * torch.arange(8, device="cuda:0")[:, None]
    x = (x.float() + 30.0 * (lift % of < every)).to(TYPES[dtype])
    _run(x, _scores(1, 8, 15), K=16)
    _run(x, _scores(1, 8, 16), K=64, done=np.array([[0, 0, 1, 0, 0, 0, 1, 1]]))
    x[:, ::3] = x[:, 1:2]                           # ... many of them equal
    _run(x, np.zeros((1, 8)), K=64)


def test_finished_beams_among_the_best_and_more_candidates_than_live_beams():
    # half of the beams are finished and lead: fewer sets of tokens reach the threshold than candidates are asked for
    x = _logits(64, 60001, "fp32", 16)
    done = np.tile([1, 0], 32).reshape(2, 32)
    _run(x, np.where(done == 1, -0.5, -3.0) - np.arange(32) * 0.01, K=40, done=done)


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_tokens(dtype):
    x = _logits(8, 20000, dtype, 7)
    x[0] = -np.inf                                  # nothing is allowed
    x[1, :] = -np.inf
    x[1, 12345] = -3.0                              # one token is
    x[2, 5:] = -np.inf
    x[3, 8192:16384] = -np.inf                      # a whole segment is not
    x[4:] = -np.inf
    x[5, 19999] = 0.5
    x[5, 0] = 0.25
    _run(x, _scores(2, 4, 7), K=8, eos=0)
    x[:] = -np.inf
    _run(x, _scores(2, 4, 7), K=8)


def test_the_types_lowest_value_is_a_candidate():
    for dtype in TYPES.values():
        x = torch.full((2, 700), torch.finfo(dtype).min, device="cuda:0", dtype=dtype)
        _run(x, np.zeros((1, 2)), K=5)
        x[:, 3] = 1.0
        x[:, 699] = torch.finfo(dtype).max if dtype != torch.float16 else 100.0
        _run(x, np.zeros((1, 2)), K=1)


def test_scores_that_fp32_does_not_hold():
    big = torch.finfo(torch.float32).max
    # logits at either end: the lowest have scores of twice the lowest number, and are no candidates
    x = torch.full((2, 900), -big, device="cuda:0")
    x[:, 5], x[:, 700] = 1.0, big
    op, dev = _op(x, np.array([[0.0, -1.0]]), 4)
    got = op.run()
    torch.cuda.synchronize()
    assert dev.read_status() == 0
    # (700: score less nothing; 5: 1 - big; the others -2 big)
    assert got["token"].tolist() == [[700, 700, 5, 5]] and got["parent"].tolist() == [[0, 1, 0, 1]]
    assert got["score"].tolist() == [[0.0, -1.0, -big, -big]]
    op, dev = _op(x, np.array([[0.0, -1.0]]), 7)
    got = op.run()
    torch.cuda.synchronize()
    assert dev.read_status() == 0 and got["token"].tolist() == [[700, 700, 5, 5, -1, -1, -1]] and got["n_new"].tolist() == [[1, 1, 1, 1, 0, 0, 0]]
    # a score that less the logarithm fits no more
    op, dev = _op(x, np.array([[-1e38, 0.0]]), 2)
    got = op.run()
    torch.cuda.synchronize()
    assert dev.read_status() == M.MEPIC_DEV_BAD_LOGITS and got["token"].tolist() == [[700, 5]] and got["parent"].tolist() == [[1, 1]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("at", [0, 9000, 19999])
def test_a_row_with_nan_or_infinity_offers_nothing(dtype, what, at):
    x = _logits(6, 20000, dtype, 9)
    x[1, at] = what
    x[3, :] = -np.inf
    x[3, at] = what
    _run(x, _scores(2, 3, 9), K=3)


def test_the_most_beams_there_may_be():
    _run(_logits(65535, 6, "bf16", 12), _scores(13107, 5, 12), K=3)


def test_scores_that_are_no_numbers():
    x = _logits(6, 3000, "bf16", 10)
    _run(x, np.array([[0.0, -np.inf, -1.0], [-np.inf, -np.inf, -np.inf]]), K=4)
    _run(x, np.array([[0.0, np.nan, -1.0], [np.inf, -2.0, -np.inf]]), K=4)
    x[1] = float("nan")                              # a row that does not count is not looked at
    _run(x, np.array([[0.0, -np.inf, -1.0], [0.0, -1.0, -2.0]]), K=4)
    _run(x, np.array([[0.0, -2.0, -1.0], [0.0, -1.0, -2.0]]), done=np.array([[0, 1, 0], [0, 0, 0]]), K=4)


def test_finished_beams():
    x = _logits(12, 5000, "fp32", 11)
    done = np.array([[1, 0, 0, 1], [1, 1, 1, 1], [0, 0, 0, 5]])
    scores = np.array([[-0.1, -3, -4, -30.0], [-4, -3, -3, -9], [-1, -1, -1, -np.inf]])
    op, _ = _run(x, scores, done=done, K=4, eos=7, pad=9)
    assert op.parent[1].tolist() == [1, 2, 0, 3] and op.token[1].tolist() == [9] * 4 and op.n_new[1].tolist() == [0] * 4
    _run(x, scores, done=done, K=8, eos=7, pad=9)                  # group 1 has four candidates for eight places


def test_captured_and_replayed_with_other_logits():
    x, sc = _logits(8, 40001, "bf16", 12), torch.from_numpy(_scores(2, 4, 12).astype(np.float32)).cuda()
    done = dev32(np.zeros((2, 4)))
    dev = RT.Device(CFG)
    op = RT.BeamSelect(dev, logits=x, scores=sc, done=done, eos_token=1)
    op.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = op.run()
    for seed in range(3):
        x.copy_(_logits(8, 40001, "bf16", 20 + seed))
        sc.copy_(torch.from_numpy(_scores(2, 4, 30 + seed).astype(np.float32)))
        done[0, seed] = 1
        graph.replay()
        torch.cuda.synchronize()
        _check(x, sc.double().cpu().numpy(), done.cpu().numpy(), 4, 1, 0, got, dev.read_status())


def test_logits_past_32_bits_of_elements():
    # three rows 2^31 elements apart
    buf = torch.empty((1 << 32) + 5000, dtype=torch.bfloat16, device="cuda:0")
    x = buf.as_strided((3, 5000), (1 << 31, 1))
    x.copy_(_logits(3, 5000, "bf16", 13))
    _run(x, _scores(1, 3, 13), K=6)


@pytest.mark.parametrize("seed", range(10))
def test_random_shapes(seed):
    rng = np.random.default_rng(seed)
    G, W = int(rng.integers(1, 9)), int(rng.integers(1, 33))
    V = int(np.exp(rng.uniform(0, np.log(70000))))
    x = _logits(G * W, V, str(rng.choice(list(TYPES))), seed, float(rng.choice([0.1, 2, 8])))
    x[torch.rand(x.shape, device="cuda:0") < 0.1] = -np.inf
    done = (rng.random((G, W)) < 0.2).astype(np.int64)
    _run(x, _scores(G, W, seed), done=done, K=int(rng.integers(1, 65)), eos=int(rng.integers(-1, V)) if V > 1 else None, pad=int(rng.integers(0, V)))
