"""What dash_attn_rope asks of its parameters: a rotation knows nothing of chunks, groups and scores.  Without a GPU a call that is
accepted ends at the device check."""
import ctypes

import pytest
import torch

from paper_2605_18753_b200 import binding as B

# (an accepted call would launch: the addresses here are none)
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host checks of calls that are accepted")


@pytest.fixture(scope="module")
def lib():
    from paper_2605_18753_b200 import build
    build.build()
    return B.lib()


def _p(**kw):
    base = dict(batch=1, seq_q=64, seq_kv=64, h_q=4, h_kv=2, head_dim=64, block=64, dtype=B.DASH_BF16, alpha=1.5)
    base.update(kw)
    base.setdefault("seq_kv", base["seq_q"])
    return B.make_params(**base)


def _call(lib, p, *args):
    r = B.make_rope([1.0, 0.5], axis=[0, 1])
    return lib.dash_attn_rope(ctypes.byref(p), ctypes.byref(r), *args, None)


def _accepted(lib, p, *args):
    return _call(lib, p, *(args or (16, 16, 16, 16, 16, 0))) not in (-1, -2, -3)


@pytest.mark.parametrize("kw", [
    dict(h_q=6, h_kv=2), dict(h_q=24, h_kv=8), dict(h_q=28, h_kv=4), dict(h_q=71, h_kv=1), dict(h_q=128, h_kv=1), dict(h_q=64, h_kv=64),
    dict(seq_q=1048576, seq_kv=1048576), dict(seq_q=600000, seq_kv=600000, block=16), dict(seq_q=1, seq_kv=1), dict(batch=3, seq_q=7, seq_kv=7),
    dict(block=48), dict(alpha=1.0), dict(gamma=0.0), dict(sigma=0.0), dict(causal=2), dict(local_blocks=-1),
    dict(v_stride=(1, 2, 3)), dict(o_stride=(-8, 8, 8)),
])
def test_parameters_of_the_attention_do_not_matter(lib, kw):
    assert _accepted(lib, _p(**kw))


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -1), (dict(batch=65536), -1), (dict(seq_q=0, seq_kv=0), -1), (dict(seq_q=1, seq_kv=64), -1), (dict(seq_q=32, seq_kv=64), -1),
    (dict(h_q=0), -1), (dict(h_kv=0), -1), (dict(h_q=5), -1), (dict(dtype=7), -1), (dict(head_dim=96), -2), (dict(q_stride=(4096, 256, 63)), -1),
    (dict(k_stride=(4096, -64, 64)), -1), (dict(k_stride=(1 << 41, 128, 64)), -1), (dict(batch=65535, seq_q=1 << 20, seq_kv=1 << 20), -2),
])
def test_what_it_needs_is_checked(lib, kw, code):
    assert _call(lib, _p(**kw), 16, 16, 16, 16, 16, 0) == code


def test_strides_of_an_absent_tensor_do_not_matter(lib):
    p = _p(k_stride=(3, 5, 7))
    assert _accepted(lib, p, 16, 16, None, 16, None, 0)
    assert _call(lib, p, 16, None, 16, None, 16, 0) == -1
    bad = _p()
    bad.struct_size = 8
    assert _call(lib, bad, 16, 16, 16, 16, 16, 0) == -1


@pytest.mark.parametrize("freq,code", [(2.0 ** 40, None), (-2.0 ** 40, None), (2.0 ** 40 * (1 + 2.0 ** -52), -1), (-1e300, -1),
                                       (float("inf"), -1), (float("nan"), -1), (0.0, None), (-1e-300, None)])
def test_frequencies_whose_fraction_is_lost_are_refused(lib, freq, code):
    got = lib.dash_attn_rope(ctypes.byref(_p()), ctypes.byref(B.make_rope([1.0, freq])), 16, 16, 16, 16, 16, 0, None)
    assert got == code if code else got not in (-1, -2, -3)
