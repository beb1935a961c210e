"""The V ring of the bf16 chunk attention under loads that come late: units of odd and even numbers of tiles, in turns and of two row
tiles, whole and cut, one behind another in a block.  Every run has to give the same bits, with and without tiles held back, and the
float64 definition's values (tolerances: test_gpu_paged_operators.py).  What lies behind the caches is NaN."""
import pytest
import torch

from paper_2605_18753_b200 import binding as B
from tests.test_gpu_paged_operators import BF, DEV, Cache

pytestmark = pytest.mark.gpu


@pytest.fixture
def held():
    yield B.dash_attn_test_hold_loads
    B.dash_attn_test_hold_loads()


def _mix(tiles, new, n, seed):
    """n sequences with caches of `tiles` tiles of 128 slots, not quite full ones, and `new` new tokens, drawn in a mixed order."""
    g = torch.Generator().manual_seed(seed)
    pick = lambda xs: [xs[int(k)] for k in torch.randint(0, len(xs), (n,), generator=g)]  # noqa: E731
    kv = [128 * t - int(torch.randint(0, 128, (1,), generator=g)) for t in pick(tiles)]
    return [min(q, k) for q, k in zip(pick(new), kv)], kv


def _one_tile_each(c, seed):
    """Every (sequence, KV head) gets its weight from one tile, another one for each: a key that its queries are drawn to."""
    g = torch.Generator().manual_seed(seed)
    group = c.h_q // c.h_kv
    for b, a, e in c.spans():
        for r in range(c.h_kv):
            slot = int(torch.randint(0, max(1, c.kv_lens[b] - (e - a)), (1,), generator=g))
            key = c.Q[a:e, r * group:(r + 1) * group].float().mean((0, 1)).cpu()
            c.Kc[b][slot, r] = (key * (c.d ** 0.5 * 8 / key.norm().clamp(min=1e-3) ** 2)).to(c.dtype)
            c.Kpool[c.table[b, slot // c.page].long(), slot % c.page, r] = c.Kc[b][slot, r].to(DEV)


CASES = [
    # (tiles of the caches, new tokens, sequences, h_q, h_kv, d)
    ([1, 3, 5], [1], 300, 4, 2, 128),               # more units than blocks: whole ones and cut ones in every block
    ([1, 2, 3, 4, 5, 10], [1, 2], 260, 8, 2, 64),
    ([3], [1], 200, 4, 4, 128),
    ([5, 2], [1, 40, 3], 150, 8, 2, 128),           # units of one row tile and of two in turn
    ([3, 4, 5, 10, 71], [1], 100, 4, 2, 128),
    ([3, 1, 4], [33, 60, 1, 20], 120, 16, 2, 64),
]


@pytest.mark.parametrize("tiles,new,n,h_q,h_kv,d", CASES)
def test_late_tiles_change_nothing(held, tiles, new, n, h_q, h_kv, d):
    q_lens, kv_lens = _mix(tiles, new, n, n)
    c = Cache(q_lens, kv_lens, h_q=h_q, h_kv=h_kv, d=d, page=64, dtype=BF, seed=n, spare=3)
    _one_tile_each(c, n)
    c.attend()
    c.check_attention()
    O, lse = c.O.clone(), c.lse.clone()
    for cycles in (3000, 12000, 40000):
        for odd in (False, True):
            held(cycles, odd)
            c.O.fill_(7.0), c.lse.fill_(7.0)
            c.attend()
            assert torch.equal(c.O, O) and torch.equal(c.lse, lse), (cycles, odd)


@pytest.mark.parametrize("clean", [True, False])
def test_every_run_gives_the_same_bits(clean):
    """Single tokens over caches whose numbers of tiles mix odd and even, hundreds of times: each result against the first, which is
    checked; with zeros behind the caches and with NaN."""
    q_lens, kv_lens = _mix([3, 4, 5, 10, 71], [1], 90, 7)
    c = Cache(q_lens, kv_lens, h_q=8, h_kv=4, d=128, page=64, dtype=BF, seed=7)
    if clean:
        for pool in (c.Kpool, c.Vpool):
            pool.nan_to_num_(0.0)
    c.attend()
    c.check_attention()
    O, lse = c.O.clone(), c.lse.clone()
    for _ in range(300):
        c.O.fill_(7.0), c.lse.fill_(7.0)
        c.attend()
        assert torch.equal(c.O, O) and torch.equal(c.lse, lse)


@pytest.mark.parametrize("length", [9 * 128 + 5, 41 * 128 + 42, 70 * 128 + 29])
def test_every_run_of_caches_with_a_tail_gives_the_same_bits(length):
    """Equal caches that end early in a tile, each run compared (the weights lie in the tiles before the last)."""
    c = Cache([1] * 12, [length] * 12, h_q=16, h_kv=8, d=128, page=64, dtype=BF, seed=length)
    c.attend()
    c.check_attention()
    O, lse = c.O.clone(), c.lse.clone()
    for _ in range(50):
        c.O.fill_(7.0), c.lse.fill_(7.0)
        c.attend()
        assert torch.equal(c.O, O) and torch.equal(c.lse, lse)
