"""The check of long contexts sees a single wrong tile (in 64 bits, no GPU needed)."""
import pytest
import torch

from tile_signal import Tiles


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("T,D,ctx,tile", [(1, 128, 150000, 128), (3, 64, 90000, 128), (2, 128, 20000, 64)])
def test_one_wrong_tile_is_seen(dtype, T, D, ctx, tile):
    p = Tiles(dtype, T, 2, 1, D, 64, [ctx], tile=tile, seed=ctx)
    want = p.reference(0)
    rounded = want[0].to(dtype)
    assert p.misses(0, rounded, want[1].float(), want) <= 0  # the right result, rounded once, passes
    tiles = (ctx + T - 1) // tile + 1
    for j in (1, 2, 3, 6, tiles // 3, tiles // 2, tiles - 2):
        plants = [("values", j, None), ("tile", j, None)]
        for back in (1, 2, 3, 6):  # a tile that was in the same place before: stages of one or both rings
            if j >= back:
                plants += [("values", j, j - back), ("keys", j, j - back)]
        for plant in plants:
            out, lse, _ = p.reference(0, plant=plant)
            # what the planted mistake changes in the result itself, whatever the log-sum-exp shows
            assert p.misses(0, out.to(dtype), want[1].float(), want) > 0, plant
