"""How the head's gradient cuts the vocabulary into pieces and each piece's inner axis into shares, on the CPU: the pieces cover
the vocabulary in whole tiles, and no share of any piece is without steps, whatever the sizes and however many rows are masked.  (An
empty share once put the thread that issues the products one accumulator behind the warps that read them.)"""
import random

import pytest

from paper_2605_14978_b200 import binding as B
from paper_2605_14978_b200 import build as build_mod

TILE, STEP, PAIRS = 256, 64, 74


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_mod.build()
    return B.load_library()


def check(T, V, D, live, dtype=B.PPOW_BF16):
    pieces, shares = B.ppow_head_plan(B.ppow_head_params(T, V, D, dtype, D, D, 1.0), live)
    at = 0
    for first, columns in pieces:
        assert first == at and columns > 0 and first % TILE == 0, (T, V, D, live, pieces)
        at += columns
    assert at == V
    tiles = [(c + TILE - 1) // TILE for _, c in pieces]
    assert max(tiles) - min(tiles) <= 1
    few = next((n for n in (16, 32, 64, 128) if T <= n), 0)
    rows = few or (T + TILE - 1) // TILE * TILE
    assert max(tiles) == 1 or rows * max(tiles) * TILE * 2 <= 512 << 20
    out = (1 if few else max(1, (live + TILE - 1) // TILE)) * ((D + TILE - 1) // TILE)
    assert 1 <= shares <= PAIRS and (shares == 1 or shares * out <= 8 * PAIRS)
    for _, columns in pieces:
        steps = (columns + STEP - 1) // STEP
        # share s of a piece takes steps [steps * s / shares, steps * (s + 1) / shares)
        assert shares == 1 or steps >= 8 * shares, (T, V, D, live, columns, shares)
        assert all(steps * s // shares < steps * (s + 1) // shares for s in range(shares))
    return pieces, shares


@pytest.mark.parametrize("T,V,D,live", [(51896, 128256, 1024, 3483), (49152, 129280, 2048, 2000), (98304, 128256, 2560, 1000),
                                        (65536, 151936, 5120, 100), (65536, 65537, 256, 65536), (32000, 262208, 512, 32000),
                                        (47872, 129280, 4096, 256), (262144, 3129, 768, 6700), (1 << 20, 128256, 4096, 1)])
def test_long_batches_with_a_short_last_piece(T, V, D, live):
    pieces, _ = check(T, V, D, live)
    assert len(pieces) > 2


@pytest.mark.parametrize("T", [1, 16, 17, 128, 129, 256, 257, 2304, 4096, 30000, 65536, 100001, 1 << 18, 1 << 20])
def test_no_share_is_empty(T):
    rng = random.Random(T)
    for V in (2, 257, 1000, 3129, 32000, 32001, 50257, 65537, 128256, 129280, 151936, 152064, 256000, 262208, 1 << 22):
        for D in (8, 256, 768, 2048, 4096, 5120, 1 << 16):
            counts = {0, 1, T // 2, T} | {min(T, 1 << rng.randrange(21)) for _ in range(3)} | {rng.randint(0, T) for _ in range(3)}
            for live in counts:
                check(T, V, D, live, rng.choice([B.PPOW_BF16, B.PPOW_F16]))


def test_odd_sizes():
    rng = random.Random(0)
    for _ in range(4000):
        T, V, D = int(2 ** rng.uniform(0, 20)), max(2, int(2 ** rng.uniform(1, 22))), 8 * max(1, int(2 ** rng.uniform(0, 13)))
        check(T, V, D, rng.randint(0, T) if rng.random() < 0.5 else min(T, int(2 ** rng.uniform(0, 20))))


def test_the_last_batch_of_the_largest_sizes_keeps_its_shares():
    # one piece, few tokens: the shares of dh are what fills the pairs
    assert check(8, 128256, 4096, 8)[1] > 1 and check(157, 32000, 1024, 126)[1] > 1
    assert check(4096, 128256, 4096, 4096)[0][1][0] == 250 * TILE


def test_refusals():
    p = B.ppow_head_params(8, 1000, 64, B.PPOW_BF16, 64, 64, 1.0)
    assert B.ppow_head_plan(p, 9)[0] == [] and B.ppow_head_plan(p, -1)[0] == []
    p.V = 1
    assert B.ppow_head_plan(p, 8)[0] == []
