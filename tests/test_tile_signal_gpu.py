"""Long contexts on the GPU, where a single stale, lost or doubled tile of keys or values would show."""
import pytest
import torch

from tile_signal import Tiles

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def check(asd, p):
    cache = p.cache(asd)
    ws = asd.attention_workspace(cache, p.T, p.Hq)
    status = torch.zeros(p.B, dtype=torch.int32, device="cuda")
    for _ in range(2):
        o = asd.tree_attention(p.q.cuda(), cache, torch.tensor(p.ctx, dtype=torch.int32, device="cuda"),
                               tree_mask=p.mask.cuda(), scale=p.scale, workspace=ws, status=status)
        assert ws.error() == 0 and not bool(status.any())
        for b in range(p.B):
            want = p.reference(b, device="cuda")
            far = p.misses(b, o["out"][b].cpu(), o["lse"][b].cpu(), want)
            assert far <= 0, f"request {b} is {far:.3g} further off than it may be"


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("page", [64, 48, 16, 20])  # boxes of 64, of 16, of 16 in small pages, 16-byte copies
@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 3, 1, 128), (7, 8, 2, 64), (26, 5, 1, 128), (61, 5, 1, 128)])
def test_ranges_of_many_tiles(asd, dtype, T, Hq, Hkv, D, page):
    """One row tile of one group, of both, and two row tiles; rings of both depths wrap many times."""
    check(asd, Tiles(dtype, T, Hq, Hkv, D, page, [150000, 20000, 90000], seed=page + T))


@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 3, 1, 128), (5, 8, 2, 64), (21, 4, 1, 96), (40, 3, 1, 128)])
def test_ranges_of_many_tiles_in_fp32(asd, T, Hq, Hkv, D):
    check(asd, Tiles(F32, T, Hq, Hkv, D, 24, [60000, 5000, 31000], tile=64, seed=T))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_many_requests_of_a_few_tiles(asd, dtype):
    """CTAs that work through several units, whole ones and pieces, one after the other."""
    g = torch.Generator().manual_seed(5)
    ctx = torch.randint(0, 1500, (200,), generator=g).tolist()
    check(asd, Tiles(dtype, 5, 8, 4, 64, 16, ctx, tile=64 if dtype == F32 else 128, seed=1))
