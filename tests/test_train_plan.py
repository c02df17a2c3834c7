"""The choices by size of the operators beside the compressed linear layer, on the CPU."""
import pytest

import plan_util as pu


@pytest.mark.parametrize("columns", [1, 37, 64, 65, 128, 129, 192, 193, 1000, 4096, 5248, 65536])
def test_a_part_runs_its_own_k_tiles(columns):
    """Every K tile of a part starts inside it, but for the first three, which the kernel sends out of range there."""
    tiles = pu.ce_part_k_tiles(columns)
    assert tiles >= 3 and 64 * tiles >= columns
    assert tiles == 3 or 64 * (tiles - 1) < columns


@pytest.mark.parametrize("tokens,d,v", [(16384, 4096, 50257), (8192, 4096, 70000), (16384, 4096, 33000), (8192, 4096, 128000)])
def test_a_short_last_piece_costs_what_it_has(tokens, d, v):
    """K tiles that the parts of all pieces run, against those that the vocabulary has: a part is rounded up once."""
    piece = (1 << 30) // (tokens * 2) // 256 * 256
    plan = pu.ce_input_gradient(tokens, d, min(piece, v))
    assert plan.tile == "256x256"
    run = pieces = 0
    for v0 in range(0, v, piece):
        columns = min(piece, v - v0)
        run += sum(pu.ce_part_k_tiles(min(plan.k_per_part, columns - k0)) for k0 in range(0, columns, plan.k_per_part))
        pieces += 1
    assert run <= -(-v // 64) + 3 * pieces
