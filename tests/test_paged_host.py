"""The operators around the paged cache without a GPU: pins of their float64 definitions, and what the C ABI refuses."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2605_18753_b200 import binding as B


@pytest.fixture(scope="module")
def lib():
    from paper_2605_18753_b200 import build
    build.build()
    return B.lib()


# ---------------------------------------------------------------- the definitions

@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_depends_on_distance_and_has_its_inverse_as_adjoint(interleaved):
    rng = np.random.default_rng(0)
    freq, axis = [1.0, 0.3, 0.01], [0, 1, 0]
    x, y = rng.standard_normal((2, 5, 2, 8))
    pos = rng.integers(-50, 50, (2, 5))
    rx, ry = (po.rotate(t, pos, freq, axis, interleaved) for t in (x, y))
    assert np.allclose((rx ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(rx[..., 6:], x[..., 6:])
    assert np.allclose(po.rotate(rx, pos, freq, axis, interleaved, inverse=True), x)
    # <R x, y> = <x, R^T y>: the backward pass is the inverse rotation
    assert np.allclose((rx * y).sum(), (x * po.rotate(y, pos, freq, axis, interleaved, inverse=True)).sum())
    # products depend on the difference of positions alone
    assert np.allclose((rx * ry).sum(-1), (po.rotate(x, pos + 7, freq, axis, interleaved) * po.rotate(y, pos + 7, freq, axis, interleaved)).sum(-1))
    # and against central differences along a direction
    f = lambda t: (po.rotate(x + t * y, pos, freq, axis, interleaved) ** 3).sum()  # noqa: E731
    grad = po.rotate(3 * rx ** 2, pos, freq, axis, interleaved, inverse=True)
    assert abs((f(1e-5) - f(-1e-5)) / 2e-5 - (grad * y).sum()) < 1e-6


def test_chunk_attention_is_torchs_masked_attention_and_weights_sum_to_the_rows():
    rng = np.random.default_rng(1)
    q_len, kv, h_q, h_kv, d = 5, 13, 6, 2, 8
    Q, K, V = rng.standard_normal((q_len, h_q, d)), rng.standard_normal((kv, h_kv, d)), rng.standard_normal((kv, h_kv, d))
    O, lse, _ = po.chunk_attention(Q, K, V, q_len, kv)
    t = lambda a, rep: torch.from_numpy(a).transpose(0, 1).repeat_interleave(rep, 0)[None]  # noqa: E731
    mask = torch.arange(kv)[None] <= torch.arange(kv - q_len, kv)[:, None]
    ref = torch.nn.functional.scaled_dot_product_attention(t(Q, 1), t(K, 3), t(V, 3), attn_mask=mask)[0].transpose(0, 1).numpy()
    assert np.allclose(O, ref)
    mass = po.key_mass(Q, K, lse, q_len, kv)
    assert np.allclose(mass.sum(), q_len * h_q) and np.allclose(mass.sum(1), q_len * 3)
    old = rng.random((h_kv, kv))
    both = po.key_mass(Q, K, lse, q_len, kv, old, decay=0.5)
    assert np.allclose(both - mass, np.where(np.arange(kv) < kv - q_len, 0.5 * old, 0.0))


def test_rows_before_the_cache_see_nothing():
    O, lse, _ = po.chunk_attention(np.ones((4, 1, 4)), np.ones((2, 1, 4)), np.ones((2, 1, 4)), 4, 2)
    assert np.isneginf(lse[:2]).all() and (O[:2] == 0).all() and np.isfinite(lse[2:]).all()


def test_eviction_keeps_ends_largest_and_lower_slots_of_equals():
    assert po.evicted([5, 1, 3, 3, 3, 2, 0], 7, 5, 1, 1).tolist() == [0, 2, 3, 4, 6]
    assert po.evicted([5, 3, 3, 3, 3, 2, 0], 7, 4, 1, 1).tolist() == [0, 1, 2, 6]
    assert po.evicted([np.nan, 0, -np.inf, np.nan, 1], 5, 3, 0, 0).tolist() == [1, 2, 4]
    assert po.evicted([1, 2], 2, 3, 1, 1).tolist() == [0, 1]


# ---------------------------------------------------------------- refusals

def _pp(**kw):
    p = B.DashPagedParams()
    p.struct_size = ctypes.sizeof(B.DashPagedParams)
    base = dict(batch=2, rows=8, h_q=8, h_kv=2, head_dim=128, dtype=B.DASH_BF16, page_size=64, max_pages=4, num_pages=9)
    base.update({k: v for k, v in kw.items() if "stride" not in k})
    for k, v in base.items():
        setattr(p, k, v)
    d, h_q, h_kv, ps = base["head_dim"], base["h_q"], base["h_kv"], base["page_size"]
    st = dict(q_stride=(h_q * d, d), o_stride=(h_q * d, d), kn_stride=(h_kv * d, d), vn_stride=(h_kv * d, d),
              k_stride=(ps * h_kv * d, h_kv * d, d), v_stride=(ps * h_kv * d, h_kv * d, d))
    st.update({k: v for k, v in kw.items() if "stride" in k and k != "struct_size"})
    for k, v in st.items():
        setattr(p, k, (ctypes.c_int64 * len(v))(*v))
    return p


def _ref(p):
    return ctypes.byref(p)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), -1), (dict(batch=70000), -1), (dict(rows=-1), -1), (dict(h_q=9), -1), (dict(dtype=5), -1), (dict(page_size=24), -1),
    (dict(page_size=0), -1), (dict(max_pages=0), -1), (dict(num_pages=0), -1), (dict(head_dim=96), -2), (dict(h_q=258), -2),
    (dict(max_pages=1 << 20), -2), (dict(q_stride=(1024, 127)), -1), (dict(k_stride=(1, 2, 3)), -1), (dict(k_stride=(-8, 8, 8)), -1),
])
def test_invalid_paged_parameters_are_refused_on_the_host(lib, kw, code):
    p = _pp(**kw)
    assert B.dash_attn_paged_workspace_bytes(p) == 0
    assert lib.dash_attn_append_paged(_ref(p), None, None, 16, 16, 16, 16, 16, 16, 16, 16, 16, None) == code
    assert lib.dash_attn_attend_chunk_paged(_ref(p), 16, 16, 16, 16, 16, 16, 16, 16, 256, 1 << 30, None) == code
    assert lib.dash_attn_key_mass_paged(_ref(p), 16, 16, 16, 16, 16, 16, 1.0, 16, 16, 256, 1 << 30, None) == code
    assert lib.dash_attn_evict_paged(_ref(p), 8, 1, 1, 16, 16, 16, 16, 16, 16, 32, 48, 4, 9, 64, 64, 16, None) == code


def test_struct_sizes_pointers_and_workspaces(lib):
    p = _pp()
    assert ctypes.sizeof(B.DashPagedParams) == 40 + 8 * 14 and ctypes.sizeof(B.DashRope) == 32
    bad = _pp()
    bad.struct_size = 8
    assert B.dash_attn_paged_workspace_bytes(bad) == 0
    need = B.dash_attn_paged_workspace_bytes(p)
    assert need > 0
    call = lambda *a: lib.dash_attn_attend_chunk_paged(_ref(p), *a, None)  # noqa: E731
    for k in range(7):
        args = [16] * 7
        args[k] = None
        assert call(*args, None, 256, need) == -1
        if k in (0, 1, 2, 6):
            args[k] = 24                                   # not 16-byte aligned
            assert call(*args, None, 256, need) == -1
    assert call(*[16] * 7, None, 128, need) == -3 and call(*[16] * 7, None, 256, need - 1) == -3 and call(*[16] * 7, None, None, need) == -3
    assert lib.dash_attn_key_mass_paged(_ref(p), 16, 16, 16, 16, 16, 16, float("nan"), None, 16, 256, need, None) == -1
    assert lib.dash_attn_key_mass_paged(_ref(p), 16, 16, 16, 16, 16, None, 1.0, None, 16, 256, need, None) == -1
    # broadcast outputs
    assert lib.dash_attn_attend_chunk_paged(_ref(_pp(o_stride=(0, 128))), *[16] * 7, None, 256, need, None) == -1
    # tensor maps have no stride of 0: bf16 pools and queries may not repeat
    assert lib.dash_attn_attend_chunk_paged(_ref(_pp(k_stride=(64 * 256, 256, 0))), *[16] * 7, None, 256, need, None) == -2
    assert lib.dash_attn_key_mass_paged(_ref(_pp(q_stride=(0, 128))), 16, 16, 16, 16, 16, 16, 1.0, None, 16, 256, need, None) == -2


def test_rope_refusals(lib):
    p = B.make_params(batch=1, seq_q=64, seq_kv=64, h_q=4, h_kv=2, head_dim=64, block=64, dtype=B.DASH_BF16, alpha=1.5)
    call = lambda r, *a, p=p: lib.dash_attn_rope(_ref(p), _ref(r), *a, None)  # noqa: E731
    ok = (16, 16, 16, 16, 16, 0)
    for r in (B.make_rope([0.1] * 33), B.make_rope([]), B.make_rope([0.1, float("inf")]), B.make_rope([0.1, 0.2], axis=[0, 4]),
              B.make_rope([0.1, 0.2], axis=[0, -1])):
        assert call(r, *ok) == -1
    r = B.make_rope([1.0, 0.5], axis=[0, 1])
    r.struct_size = 4
    assert call(r, *ok) == -1
    r = B.make_rope([1.0, 0.5], axis=[0, 1])
    assert call(r, None, 16, 16, 16, 16, 0) == -1                # no positions
    assert call(r, 16, None, None, None, None, 0) == -1          # nothing to rotate
    assert call(r, 16, 16, None, None, None, 0) == -1            # no output
    assert call(r, 16, 24, None, 16, None, 0) == -1              # alignment
    assert call(r, 16, 16, None, 16, None, 2) == -1              # inverse is 0 or 1
    dec = B.make_params(batch=1, seq_q=1, seq_kv=64, h_q=4, h_kv=2, head_dim=64, block=64, dtype=B.DASH_BF16, alpha=1.5)
    assert call(r, *ok, p=dec) == -1
    exp = B.make_params(batch=2, seq_q=64, seq_kv=64, h_q=4, h_kv=2, head_dim=64, block=64, dtype=B.DASH_BF16, alpha=1.5, q_stride=(0, 256, 64))
    assert call(r, *ok, p=exp) == -1                             # a broadcast output
    with pytest.raises(ValueError):
        B.make_rope([1.0, 2.0], axis=[0])


def test_append_and_evict_refusals(lib):
    p = _pp()
    r = B.make_rope([1.0, 0.5])
    app = lambda *a, p=p: lib.dash_attn_append_paged(_ref(p), *a, None)  # noqa: E731
    assert app(_ref(r), None, 16, 16, 16, 16, 16, 16, 16, 16, 16) == -1             # rope without positions
    assert app(None, 16, 16, 16, 16, 16, 16, 16, 16, 16, 16) == -1                  # positions without rope
    assert app(None, None, 16, 16, 16, 16, None, 16, 16, 16, 16) == -1              # Q without Qout
    assert app(None, None, 16, 16, 16, 16, 16, 16, 16, 16, 16, p=_pp(o_stride=(1032, 128))) == -1      # in place, other strides
    assert app(None, None, 16, 16, 16, None, None, 16, 16, 16, 16, p=_pp(v_stride=(0, 256, 128))) == -1
    ev = lambda keep, sinks, recent, *a, p=p: lib.dash_attn_evict_paged(_ref(p), keep, sinks, recent, *a, None)  # noqa: E731
    good = [16, 32, 48, 64, 64, 80, 96, 112, 4, 9, 128, 128, 144]
    for keep, sinks, recent in ((0, 0, 0), (8, -1, 0), (8, 0, -1), (8, 5, 4)):
        assert ev(keep, sinks, recent, *good) == -1
    for k in (0, 1, 2, 3, 4, 5, 6, 7, 10, 11):
        assert ev(8, 1, 1, *[None if i == k else v for i, v in enumerate(good)]) == -1
    assert ev(200, 1, 1, *good[:8], 3, *good[9:]) == -1                             # destination table too narrow
    same = list(good)
    same[6] = same[1]
    assert ev(8, 1, 1, *same) == -1                                                 # new_len is kv_len
    half = list(good)
    half[7] = half[2]
    assert ev(8, 1, 1, *half) == -1                                                 # the same table, other pools
    own = list(good)
    own[12] = own[0]
    assert ev(8, 1, 1, *own) == -1                                                  # mass in place, tokens elsewhere


def test_binding_refuses_wrong_shapes_and_types():
    pool = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    table = torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.params_for_paged(pool, pool.float(), table, h_q=4)
    with pytest.raises(ValueError):
        B.params_for_paged(pool, pool, table, h_q=4, Q=torch.zeros(5, 4, 64))
    with pytest.raises(ValueError):
        B.params_for_paged(pool, pool, table, h_q=4, Q=torch.zeros(5, 2, 64, dtype=torch.bfloat16))
    p = B.params_for_paged(pool, None, table, h_q=4, rows=0)
    assert (p.batch, p.rows, p.page_size, p.max_pages, p.num_pages) == (1, 0, 16, 2, 3)


def test_binding_refuses_sizes_that_do_not_fit_the_parameters(monkeypatch):
    """What a kernel would write or read past the end of is refused before the library is called (tensors of the CPU here, taken for
    those of the current device)."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: pytest.fail("the call went through"), raising=False)
    bf, i32 = torch.bfloat16, torch.int32
    K, V = torch.zeros(5, 16, 2, 64, dtype=bf), torch.zeros(5, 16, 2, 64, dtype=bf)
    table, q_start, kv_len = torch.zeros(3, 4, dtype=i32), torch.zeros(4, dtype=i32), torch.zeros(3, dtype=i32)
    Q, kn, pos = torch.zeros(6, 4, 64, dtype=bf), torch.zeros(6, 2, 64, dtype=bf), torch.zeros(1, 6, dtype=i32)
    lse, mass, ws = torch.zeros(6, 4), torch.zeros(3, 2, 64), torch.zeros(1, dtype=torch.uint8)
    kept, new_len = torch.zeros(3, 2, 8, dtype=i32), torch.zeros(3, dtype=i32)
    p = B.params_for_paged(K, V, table, h_q=4, Q=Q, O=Q)
    rope = B.make_rope([1.0] * 32)
    args = {
        "append": dict(rope=rope, positions=pos, q_start=q_start, kv_len=kv_len, page_table=table, Q=Q, Qout=Q, K=kn, V=kn, Kpool=K, Vpool=V),
        "attend_chunk": dict(Q=Q, Kpool=K, Vpool=V, page_table=table, q_start=q_start, kv_len=kv_len, O=Q, lse=lse, workspace=ws),
        "key_mass": dict(Q=Q, Kpool=K, page_table=table, q_start=q_start, kv_len=kv_len, lse=lse, mass_in=mass, mass_out=mass, workspace=ws),
        "evict": dict(mass=mass, kv_len=kv_len, page_table=table, Kpool=K, Vpool=V, kept=kept, new_len=new_len, dst_table=table, Kdst=K,
                      Vdst=V, mass_out=mass, keep=8),
    }
    for name, kw in args.items():
        call = getattr(B, f"dash_attn_{name}_paged")
        for arg, t in kw.items():
            if arg in ("rope", "workspace", "keep") or (name == "evict" and arg in ("Kdst", "dst_table")):
                continue
            short = t[..., :-1].contiguous() if t.dim() == 1 else t[:-1].contiguous()
            if arg == "positions":
                short = t[:, :-1].contiguous()
            with pytest.raises(ValueError):
                call(p, **{**kw, arg: short})
    with pytest.raises(ValueError):
        B.dash_attn_append_paged(p, **{**args["append"], "rope": None})
    with pytest.raises(ValueError):
        B.dash_attn_append_paged(p, **{**args["append"], "positions": None})
    with pytest.raises(ValueError):
        B.dash_attn_evict_paged(p, **{**args["evict"], "dst_table": table[:2].contiguous()})
    with pytest.raises(ValueError):
        B.dash_attn_evict_paged(p, **{**args["evict"], "Kdst": K[:4].contiguous()})
    x = torch.zeros(2, 8, 4, 64, dtype=bf)
    rp = B.params_for_prefill(x, x[:, :, :2].contiguous(), x[:, :, :2].contiguous(), x, block=16, alpha=1.5)
    pos = torch.zeros(1, 2, 8, dtype=i32)
    for a, b in ((x, x[:, :7].contiguous()), (x[:1].contiguous(), x[:1].contiguous()), (x[:, :7].contiguous(), x[:, :7].contiguous())):
        with pytest.raises(ValueError):
            B.dash_attn_rope(rp, rope, pos, a, None, b, None)
