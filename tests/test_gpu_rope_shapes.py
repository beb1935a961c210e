"""Rotary positions at head groups and lengths that the routed attention does not take (tolerances: test_gpu_paged_operators.py)."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2605_18753_b200 import binding as B
from tests.test_gpu_paged_operators import BF, DEV, F32, np64, rope_tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("h_q,h_kv,d,batch,n,block", [
    (6, 2, 64, 2, 33, 64), (24, 8, 128, 1, 70, 64), (28, 4, 128, 1, 5, 16), (71, 1, 64, 1, 9, 64), (128, 1, 64, 3, 2, 128), (9, 3, 64, 1, 1, 48)])
def test_groups_of_any_size(dtype, h_q, h_kv, d, batch, n, block):
    g = torch.Generator().manual_seed(h_q)
    Q, K = (torch.randn(batch, n, h, d, generator=g).to(dtype).to(DEV) for h in (h_q, h_kv))
    pos = torch.randint(-1000, 100000, (2, batch, n), generator=g).to(torch.int32).to(DEV)
    freq, axis = [10000.0 ** (-2 * i / d) for i in range(d // 2)], [i % 2 for i in range(d // 2)]
    p = B.make_params(batch=batch, seq_q=n, seq_kv=n, h_q=h_q, h_kv=h_kv, head_dim=d, block=block, dtype=dtype, alpha=1.5)
    for inverse in (False, True):
        Qo, Ko = torch.full_like(Q, 7.0), torch.full_like(K, 7.0)
        B.dash_attn_rope(p, B.make_rope(freq, axis=axis), pos, Q, K, Qo, Ko, inverse=inverse)
        for x, got in ((Q, Qo), (K, Ko)):
            flat = np64(x).reshape(batch * n, -1, d)
            ref = po.rotate(flat, pos.cpu().numpy().reshape(2, -1), freq, axis, False, inverse)
            assert (np.abs(np64(got).reshape(flat.shape) - ref) <= rope_tolerance(flat, ref, dtype, d // 2, False)).all()


@pytest.mark.parametrize("n,block", [(1048576, 64), (600000, 16)])
def test_long_sequences(n, block):
    g = torch.Generator(device=DEV).manual_seed(n)
    x = torch.randn(1, n, 1, 64, generator=g, device=DEV).to(BF)
    pos = torch.arange(n, dtype=torch.int32, device=DEV).view(1, 1, n)
    freq = [500000.0 ** (-i / 32) for i in range(32)]
    p = B.make_params(batch=1, seq_q=n, seq_kv=n, h_q=1, h_kv=1, head_dim=64, block=block, dtype=BF, alpha=1.5)
    out = torch.full_like(x, 7.0)
    B.dash_attn_rope(p, B.make_rope(freq), pos, x, None, out, None)
    at = torch.cat([torch.arange(5), torch.arange(n // 2, n // 2 + 300), torch.arange(n - 70, n)])
    flat = np64(x[0, at.to(DEV)])
    ref = po.rotate(flat, at.numpy()[None], freq, [0] * 32)
    assert (np.abs(np64(out[0, at.to(DEV)]) - ref) <= rope_tolerance(flat, ref, BF, 32, False)).all()
    back = torch.empty_like(x)
    B.dash_attn_rope(p, B.make_rope(freq), pos, out, None, back, None, inverse=True)
    # twice half a step of values that a rotation leaves below their pair's length, and the sums' own error
    a = x.float().abs()
    length = a + a.roll(32, -1)
    assert ((back.float() - x.float()).abs() <= 2.0 ** -8 * 2.1 * length).all()
