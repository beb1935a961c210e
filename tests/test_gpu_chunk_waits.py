"""Waits that nothing will ever satisfy, in the middle of a block's work: through the test hooks a K tile is never loaded and a wait gives
up after 2e5 clocks (0.1 ms).  Products and copies in flight end, tensor memory is freed, the kernel returns with DASH_ERR_TIMEOUT in
the status word, and after a reset the workspace serves the same bits again."""
import time

import pytest
import torch

from paper_2605_18753_b200 import binding as B
from tests.test_gpu_paged_operators import BF, DEV, Cache

pytestmark = pytest.mark.gpu
DASH_ERR_TIMEOUT = -7


@pytest.mark.parametrize("q_lens,kv_lens,d", [([1] * 8, [4000 + 130 * k for k in range(8)], 128), ([300, 40], [9000, 5000], 128),
                                              ([700, 1, 1], [4000, 9000, 300], 64)])
def test_waits_run_out_and_the_kernels_return(q_lens, kv_lens, d):
    c = Cache(q_lens, kv_lens, h_q=32, h_kv=8, d=d, page=64, dtype=BF, q_scale=1.0)
    out = torch.zeros(len(q_lens), 8, c.cap, device=DEV)
    attend = lambda: B.dash_attn_attend_chunk_paged(c.p, c.Q, c.Kpool, c.Vpool, c.table, c.q_start, c.kv_len, c.O, c.lse, c.ws)  # noqa: E731
    weigh = lambda: B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, None, out, c.ws)  # noqa: E731
    c.attend()
    weigh()
    assert B.dash_attn_last_status(c.ws) == 0
    good = [t.clone() for t in (c.O, c.lse, out)]
    for call in (attend, weigh):
        try:
            B.dash_attn_test_hooks(wait_limit_cycles=200_000, skip_own_k_load=1)
            t0 = time.time()
            call()
            assert B.dash_attn_last_status(c.ws) == DASH_ERR_TIMEOUT
            assert time.time() - t0 < 5.0
        finally:
            B.dash_attn_test_hooks()
        torch.cuda.synchronize()
        B.dash_attn_reset_status(c.ws)
        c.attend()
        weigh()
        assert B.dash_attn_last_status(c.ws) == 0
        assert all(torch.equal(a, b) for a, b in zip(good, (c.O, c.lse, out)))
