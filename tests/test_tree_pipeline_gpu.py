"""Attention of drafted rows where every CTA takes many key tiles: rings that wrap, items that follow one another in a CTA, and
references that move in the middle of an item."""
import numpy as np
import pytest
import torch

from paper_2512_16822_b200 import runtime as RT
from paper_2512_16822_b200.build import build_library
from mepic_inputs import bf16_bits_to_f64, f32_to_bf16_bits
from oracle import mepic_oracle as O
from tree_helpers import TreeCase, dev32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"


def tiles_per_cta(case):
    """Key tiles (128 keys) times row tiles (128 / G drafted rows) of all items over the multiprocessors: a CTA each."""
    row_tiles = -(-case.rows // (128 // (case.Hq // case.Hkv)))
    key_tiles = -(-case.kv_len.astype(np.int64) // 128) + -(-case.rows // 128)
    return float((row_tiles * key_tiles).sum() * case.Hkv / torch.cuda.get_device_properties(0).multi_processor_count)


def page_amplitudes(case, k_least, v_least, v_most):
    """Every page (and kv head) gets a magnitude of its own, so that another page's scale in its place would show: K's are
    2^k_least .. 1 (scores stay of order 1), V's 2^v_least .. 2^v_most."""
    shape = (case.num_pages, case.Hkv, 1, 1)
    for name, lo, hi in (("kp", k_least, 0), ("vp", v_least, v_most)):
        x = bf16_bits_to_f64(getattr(case, name)) * 2.0 ** case.rng.uniform(lo, hi, size=shape)
        setattr(case, name, f32_to_bf16_bits(x.astype(np.float32)))


def run_and_check(case, sm_scale, least_tiles, which=None):
    assert tiles_per_cta(case) >= least_tiles
    case.device()
    batch = case.batch()
    out = batch.run(sm_scale)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    case.check(out, sm_scale, which=which)
    first = out.clone()
    for _ in range(3):
        batch.run(sm_scale)
    torch.cuda.synchronize()
    assert torch.equal(batch.out, first)


@pytest.mark.parametrize("fp8", [False, True])
def test_many_short_items_in_a_cta(fp8):
    # several items (segments) per CTA, of one to six context tiles and a tile of drafted rows each
    rng = np.random.default_rng(100)
    specs = [(int(rng.integers(0, 700)), int(rng.integers(0, 8))) for _ in range(70)]
    case = TreeCase(100, Hq=16, Hkv=8, D=128, P=16, specs=specs, fp8=fp8)
    page_amplitudes(case, -3, -3, 3)
    run_and_check(case, 1.0 / np.sqrt(128), 10)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("P", [16, 64])
def test_long_items_in_a_cta(fp8, P):
    # about 20 tiles per CTA, few items: stages, scale rings and barriers wrap many times within an item
    case = TreeCase(101 + P, Hq=8, Hkv=8, D=128, P=P, specs=[(20003, 2), (19000, 3), (9777, 1), (128, 4)], theta=5e5, fp8=fp8)
    page_amplitudes(case, -3, -3, 3)
    run_and_check(case, 1.0 / np.sqrt(128), 20)


@pytest.mark.parametrize("fp8", [False, True])
def test_several_row_tiles_and_long_contexts(fp8):
    # two and three row tiles per request (levels of the cut), a drafted tile behind the context in every one
    case = TreeCase(103, Hq=16, Hkv=4, D=128, P=32, specs=[(5000, 40), (3001, 70), (4096, 33)], fp8=fp8)
    page_amplitudes(case, -3, -3, 3)
    run_and_check(case, 1.0 / np.sqrt(128), 6, which=[0])


def test_narrow_heads():
    case = TreeCase(104, Hq=16, Hkv=8, D=64, P=16, specs=[(9001, 3), (12000, 2), (40, 20), (700, 70)])
    page_amplitudes(case, -3, -3, 3)
    run_and_check(case, 0.125, 9)


@pytest.mark.parametrize("seed", range(10))
def test_random_shapes_of_many_tiles(seed):
    rng = np.random.default_rng(2000 + seed)
    Hkv = int(rng.choice([2, 3, 8]))
    G = int(rng.integers(1, 9))
    fp8 = bool(seed % 2)
    D = 128 if fp8 else int(rng.choice([64, 128]))
    P = int(rng.choice([16, 32, 64, 256]))
    specs = []
    while not specs or sum(-(-n // (128 // G)) * (-(-k // 128) + -(-n // 128)) for k, n in specs) * Hkv < 5 * 148:
        specs.append((int(rng.choice([0, 1, 128, int(rng.integers(1, 3000)), int(rng.integers(1, 12000))])), int(rng.choice([0, 1, int(rng.integers(1, 30))]))))
    case = TreeCase(3000 + seed, Hq=Hkv * G, Hkv=Hkv, D=D, P=P, specs=specs, kind=str(rng.choice(["tree", "chain", "star"])), fp8=fp8, theta=5e5)
    page_amplitudes(case, -3, -3, 3)
    # the oracle looks at the requests that cost it little, three at least
    cost = case.rows * (case.kv_len + case.rows) * case.Hq
    order = [int(b) for b in np.argsort(cost) if case.rows[b]]
    run_and_check(case, 1.0 / np.sqrt(D), 4, which=[b for i, b in enumerate(order) if i < 3 or cost[b] < 400_000])


# Scores that are whole numbers in base 2: q and K are zero but in one pair of dims that no position here turns by more than
# 1e-4 rad (its partner is zero, so the rotated element is the element), sm_scale is ln 2, and every K is a value that both
# bf16 and e4m3 under a power of two hold exactly.  Then Q', K' and P are exact, and what is left is arithmetic in fp32.
LEVELS = [(0, 9), (11, 20), (22, 32), (36, 48), (52, 64)]
LN2 = float(np.float32(np.log(2.0)))


def staircase(case, rng):
    """Context scores of every (request, kv head): pairs of tiles, one with all keys at a level, one with a single key 9 to 12
    above it (so that both count), pair above pair up to a peak that lies elsewhere in every head; low ever after."""
    D, Hkv, P = case.D, case.Hkv, case.P
    kp = np.zeros((case.num_pages, Hkv, P, D))
    for b, n in enumerate(case.kv_len):
        tiles = -(-int(n) // 128)
        for h in range(Hkv):
            level = np.zeros(int(n))
            start = int(rng.integers(0, max(1, tiles - 2 * len(LEVELS))))
            for i, (low, high) in enumerate(LEVELS[:int(rng.integers(1, len(LEVELS) + 1))]):
                lo = (start + 2 * i) * 128
                level[lo:lo + 128] = low
                if lo + 128 < n:
                    level[lo + 128 + int(rng.integers(0, min(128, int(n) - lo - 128)))] = high
            for t in range(int(n)):
                kp[case.page_ids[b, t // P], h, t % P, D // 2 - 1] = level[t]
    case.kp = f32_to_bf16_bits(kp.astype(np.float32))
    assert np.array_equal(bf16_bits_to_f64(case.kp), kp)
    sign = rng.choice([1.0, 1.0, -1.0], size=case.q.shape[:2])        # for -1 the staircase goes down
    q = np.zeros(case.q.shape)
    q[..., D // 2 - 1] = sign
    case.q = f32_to_bf16_bits(q.astype(np.float32))
    kn = np.zeros(case.kn.shape)
    kn[..., D // 2 - 1] = rng.choice([0.0, 9.0, 20.0, 64.0], size=case.kn.shape[:2])
    case.kn = f32_to_bf16_bits(kn.astype(np.float32))


@pytest.mark.parametrize("D,fp8", [(128, False), (64, False), (128, True)])
def test_references_that_rise_in_the_middle_of_an_item(D, fp8):
    rng = np.random.default_rng(110 + D)
    specs = [(int(n), int(r)) for n, r in zip(rng.integers(1300, 3000, size=8), rng.integers(1, 6, size=8))]
    case = TreeCase(110 + D, Hq=16, Hkv=8, D=D, P=16, specs=specs, jitter=False, theta=1e12)
    staircase(case, rng)
    assert tiles_per_cta(case) >= 5
    case.device()
    if fp8:
        # codes and scales made here, so that they are exact: a power of two per (page, kv head)
        case.fp8 = True
        ks = 2.0 ** rng.integers(-1, 3, size=(case.num_pages, case.Hkv))
        vs = 2.0 ** rng.integers(-4, 4, size=(case.num_pages, case.Hkv))
        kc = O.e4m3_encode((bf16_bits_to_f64(case.kp) / ks[:, :, None, None]).astype(np.float32))
        vc = O.e4m3_encode(rng.standard_normal(case.vp.shape).astype(np.float32))
        assert np.array_equal(O.dequantize_pages(kc, ks.astype(np.float32)), bf16_bits_to_f64(case.kp))
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        case.pools = RT.Fp8Pools.over(case.dev, up(kc), up(vc), up(ks.astype(np.float32)), up(vs.astype(np.float32)))
    out = case.batch().run(LN2)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    got = bf16_bits_to_f64(RT.bf16_bits(out))
    kp, vp = (case.kp, case.vp) if not fp8 else (O.dequantize_pages(kc, ks.astype(np.float32)), O.dequantize_pages(vc, vs.astype(np.float32)))
    for b in range(len(specs)):
        r = slice(case.off[b], case.off[b + 1])
        want, _ = O.tree_attention_one(case.q[r], case.kn[r], case.vn[r], case.row_pos[b], case.sees[b], kp, vp, case.page_ids[b],
                                       case.pos_base[b], int(case.kv_len[b]), LN2, case.theta)
        mean, _ = O.tree_attention_one(case.q[r], case.kn[r], f32_to_bf16_bits(np.abs(bf16_bits_to_f64(case.vn[r])).astype(np.float32)), case.row_pos[b], case.sees[b],
                                       kp, np.abs(vp if fp8 else bf16_bits_to_f64(vp)), case.page_ids[b], case.pos_base[b], int(case.kv_len[b]), LN2, case.theta)
        # the output's own rounding (2^-8 relative), and fp32 on the way: every weight, sum and product is off by at most 2^-21 of
        # its value for the exponential and by 2^-23 for each of the n sums it passes through, relative to sum w |v|
        n = int(case.kv_len[b] + case.rows[b])
        tol = 2.0 ** -8 * np.abs(want) + (2 * 2.0 ** -21 + 2 * n * 2.0 ** -23) * mean
        err = np.abs(got[r] - want)
        assert (err <= tol).all(), (b, float((err / tol).max()), np.argwhere(err > tol)[:4].tolist())


@pytest.mark.parametrize("Hkv", [1, 8])              # a key tile per CTA, and several
@pytest.mark.parametrize("D", [128, 64])
def test_what_is_not_finite_shows_however_small_its_weight(D, Hkv):
    # every row sees every context slot: a NaN or an infinity among their V cannot leave a finite output, also where the weight,
    # 2^-200 here, is no fp32 number, and whichever CTA meets it.  The same for a drafted row that is seen.
    case = TreeCase(120 + D, Hq=Hkv, Hkv=Hkv, D=D, P=16, specs=[(3000, 3), (2500, 2)], jitter=False, theta=1e12, kind="star")
    case.q[:], case.kp[:], case.kn[:] = 0, 0, 0
    pair = D // 2 - 1
    case.q[..., pair] = f32_to_bf16_bits(np.float32([1.0]))[0]
    high = f32_to_bf16_bits(np.float32([200.0]))[0]
    for b, n in enumerate(case.kv_len):
        for t in range(600, int(n)):
            case.kp[case.page_ids[b, t // 16], :, t % 16, pair] = high
    odd = {3: 0x7fc0, 7: 0x7f80, 40: 0xff80}
    for d, bits in odd.items():
        case.vp[case.page_ids[0, 2], :, 5, d] = bits                    # context slot 37 of the first request
        case.vn[case.off[1], :, d] = bits                               # its first drafted row in the second
    case.device()
    out = case.batch().run(LN2)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0
    got = bf16_bits_to_f64(RT.bf16_bits(out))
    bad = np.zeros(got.shape, dtype=bool)
    bad[:case.off[1], :, list(odd)] = True
    bad[case.off[1], :, list(odd)] = True                               # a star: the other drafted row does not see that one
    assert np.array_equal(~np.isfinite(got), bad)
    assert np.isnan(got[:case.off[1] + 1, :, 3]).all()


@pytest.mark.parametrize("B", [2, 40])               # the cut by one warp, and by the CTA
def test_rows_that_no_request_owns_at_all(B):
    case = TreeCase(130, Hq=4, Hkv=1, D=128, P=16, specs=[(100, 3)] + [(50, 0)] * (B - 1))
    case.device()
    q, k, v = (RT.bf16_tensor(x, "cuda:0") for x in (case.q, case.kn, case.vn))
    batch = RT.TreeBatch(case.dev, q=q, k_new=k, v_new=v, row_offsets=dev32([0] * (B + 1)), row_pos=dev32(np.concatenate(case.row_pos)),
                         tree_mask=dev32(case.mask()), page_ids=dev32(case.page_ids), pos_base=dev32(case.pos_base), kv_len=dev32(case.kv_len), max_rows=3)
    batch.out.fill_(7.0)
    batch.run(0.09)
    torch.cuda.synchronize()
    assert case.dev.read_status() == 0 and (batch.out == 7.0).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_requests_that_alias_long_chunks_at_positions_of_their_own(fp8):
    # 150 pages that six requests share, in another order and at other positions in each, before pages of their own
    rng = np.random.default_rng(140)
    case = TreeCase(140, Hq=16, Hkv=8, D=128, P=16, specs=[(int(n), int(r)) for n, r in zip(rng.integers(2450, 3500, size=6), (1, 5, 2, 9, 1, 3))],
                    fp8=fp8, theta=5e5)
    page_amplitudes(case, -3, -3, 3)
    common = case.page_ids[0, :150].copy()
    for b in range(1, 6):
        case.page_ids[b, :150] = rng.permutation(common) if b % 2 else common
    assert len({tuple(case.pos_base[b, :150]) for b in range(6)}) == 6
    run_and_check(case, 1.0 / np.sqrt(128), 7)
