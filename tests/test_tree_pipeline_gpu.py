"""Attention of drafted rows where every CTA takes many key tiles: rings that wrap, and items that follow one another in a CTA."""
import numpy as np
import pytest
import torch

from paper_2512_16822_b200.build import build_library
from mepic_inputs import bf16_bits_to_f64, f32_to_bf16_bits
from tree_helpers import TreeCase

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

