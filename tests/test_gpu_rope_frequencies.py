"""Angles of negative and tiny frequencies at far positions.  The header's word: within 2^-31 turns at every int32 position, 2.9e-9
radians.  With the pair (1, 0) the outputs are the cosine and the sine themselves.  To the angle's error come the polynomials' (2e-9) and fp32
roundings, at most 5 * 2^-24 of the value: of the fraction made a float, the factor 2 pi / 2^32 and the product with it (each once in the
sine; in the cosine times a tan a <= 0.8), the last step, and less than one of all others together."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2605_18753_b200 import binding as B

pytestmark = pytest.mark.gpu
FREQS = [sign * f for sign in (1.0, -1.0) for f in (1.0, 0.1, 1e-2, 3.3e-4, 1e-5, 7e-8, 3e-10, 2e-13, 3.4e-16, 9e-17, 1e-18, 3.0, 12.5, 1000.1, 1e6, 2.0 ** 39)]
FAR = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, -(2 ** 30) - 54321, 1999999943, -1999999943, 131071]


@pytest.mark.parametrize("inverse", [False, True])
def test_angles_are_exact_for_both_signs(inverse):
    n = len(FAR)
    x = torch.zeros(1, n, 1, 64, device="cuda")
    x[..., :32] = 1.0
    p = B.make_params(batch=1, seq_q=n, seq_kv=n, h_q=1, h_kv=1, head_dim=64, block=64, dtype=torch.float32, alpha=1.5)
    pos = torch.tensor(FAR, dtype=torch.int64).to(torch.int32).view(1, 1, n).cuda()
    out = torch.empty_like(x)
    assert len(FREQS) == 32
    B.dash_attn_rope(p, B.make_rope(FREQS), pos, x, None, out, None, inverse=inverse)
    ref = exact(np.array(FAR), FREQS, inverse)
    err = np.abs(out[0, :, 0].double().cpu().numpy() - ref)
    tol = 2.9e-9 + 2e-9 + 5 * 2.0 ** -24 * np.abs(ref)
    assert (err <= tol).all(), [(FAR[i], FREQS[k % 32], err[i, k]) for i, k in zip(*np.nonzero(err > tol))]


def exact(positions, freqs, inverse):
    """cos and sin of position * frequency, the product taken modulo 2 pi in rational arithmetic (pi to 60 digits)."""
    from fractions import Fraction
    two_pi = 2 * Fraction(31415926535897932384626433832795028841971693993751058209749445923, 10 ** 64)
    out = np.zeros((len(positions), 64))
    for i, t in enumerate(positions):
        for k, f in enumerate(freqs):
            turns = Fraction(int(t)) * Fraction(f) / two_pi
            theta = 2 * np.pi * float(turns - round(turns))
            out[i, k], out[i, 32 + k] = np.cos(theta), np.sin(-theta if inverse else theta)
    return out


def test_the_reference_here_agrees_with_the_oracle():
    pos = np.array([5, -77, 40000])
    x = np.zeros((3, 1, 64))
    x[..., :32] = 1.0
    freqs = [0.5 ** i * (-1) ** i for i in range(32)]
    assert np.abs(po.rotate(x, pos[None], freqs, [0] * 32)[:, 0] - exact(pos, freqs, False)).max() < 1e-13
