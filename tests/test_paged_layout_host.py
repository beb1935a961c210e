"""The binding of the operators around the paged cache compares every tensor's layout with the parameters before the library is called
(tensors of the CPU here, taken for those of the current device): the kernels go by the parameters' sizes and strides, so a tensor of another
layout would be misread, or read and written past its end."""
import ctypes

import pytest
import torch

from paper_2605_18753_b200 import binding as B

BF, I32 = torch.bfloat16, torch.int32


class Called(Exception):
    pass


class Far(torch.Tensor):
    """A tensor of another device."""

    def get_device(self):
        return 5


@pytest.fixture(autouse=True)
def cpu_as_device(monkeypatch):
    def called(dev):
        raise Called
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", called, raising=False)


def _paged(rows=6, h_q=4, h_kv=2, d=64, page=16, pages=5, batch=3, width=4):
    K, V = torch.zeros(pages, page, h_kv, d, dtype=BF), torch.zeros(pages, page, h_kv, d, dtype=BF)
    table, q_start, kv_len = torch.zeros(batch, width, dtype=I32), torch.zeros(batch + 1, dtype=I32), torch.zeros(batch, dtype=I32)
    Q, kn, vn, O = (torch.zeros(rows, h, d, dtype=BF) for h in (h_q, h_kv, h_kv, h_q))
    pos, lse, mass = torch.zeros(1, rows, dtype=I32), torch.zeros(rows, h_q), torch.zeros(batch, h_kv, width * page)
    ws = torch.zeros(1, dtype=torch.uint8)
    kept, new_len, Kd, Vd = torch.zeros(batch, h_kv, 8, dtype=I32), torch.zeros(batch, dtype=I32), K.clone(), V.clone()
    calls = {
        "append": dict(rope=B.make_rope([1.0] * 32), positions=pos, q_start=q_start, kv_len=kv_len, page_table=table, Q=Q, Qout=O, K=kn, V=vn,
                       Kpool=K, Vpool=V),
        "attend_chunk": dict(Q=Q, Kpool=K, Vpool=V, page_table=table, q_start=q_start, kv_len=kv_len, O=O, lse=lse, workspace=ws),
        "key_mass": dict(Q=Q, Kpool=K, page_table=table, q_start=q_start, kv_len=kv_len, lse=lse, mass_in=mass, mass_out=mass.clone(), workspace=ws),
        "evict": dict(mass=mass, kv_len=kv_len, page_table=table, Kpool=K, Vpool=V, kept=kept, new_len=new_len, dst_table=table.clone(), Kdst=Kd,
                      Vdst=Vd, mass_out=None, keep=8),
    }
    return B.params_for_paged(K, V, table, h_q=h_q, Q=Q, O=O, K=kn, V=vn), calls


LAYOUTS = {"append": ["Q", "Qout", "K", "V", "Kpool", "Vpool"], "attend_chunk": ["Q", "O", "Kpool", "Vpool"], "key_mass": ["Q", "Kpool"],
           "evict": ["Kpool", "Vpool", "Kdst", "Vdst"]}
CASES = [(name, arg) for name, args in LAYOUTS.items() for arg in args]


def _others(t, pool):
    """Tensors of other layouts that the parameters do not describe: heads, head_dim, page size, strides of the same shape."""
    yield t[..., :-1, :].contiguous()
    yield t[..., :32].contiguous()
    wide = torch.zeros(*t.shape[:-2], t.shape[-2] + 2, t.shape[-1], dtype=t.dtype)
    yield wide[..., 1:-1, :]                                            # a slice of a fused projection, or of a wider pool
    yield t.transpose(-3, -2).contiguous().transpose(-3, -2)            # heads before tokens in memory
    yield t[..., :1, :].expand(t.shape)
    yield torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype)[..., ::2]
    yield t.flatten(-2)
    if pool:
        yield t[:, :8].contiguous()
        yield torch.cat([t, t], 1)


@pytest.mark.parametrize("name,arg", CASES)
def test_a_layout_that_the_parameters_do_not_have_is_refused(name, arg):
    p, calls = _paged()
    call = getattr(B, f"dash_attn_{name}_paged")
    with pytest.raises(Called):
        call(p, **calls[name])
    for other in _others(calls[name][arg], "pool" in arg or "dst" in arg):
        with pytest.raises(ValueError):
            call(p, **{**calls[name], arg: other})
    with pytest.raises(Called):                                         # and as before behind a refusal
        call(p, **calls[name])


@pytest.mark.parametrize("name,arg", [(n, a) for n, a in CASES if a not in ("Kdst", "Vdst")])
def test_parameters_for_another_layout_are_refused(name, arg):
    """The other way round: the tensors stay, the parameters were made for slices of wider ones, or changed since."""
    p, calls = _paged()
    field = {"Q": "q_stride", "Qout": "o_stride", "O": "o_stride", "K": "kn_stride", "V": "vn_stride", "Kpool": "k_stride", "Vpool": "v_stride"}[arg]
    call = getattr(B, f"dash_attn_{name}_paged")
    with pytest.raises(Called):
        call(p, **calls[name])
    old = list(getattr(p, field))
    getattr(p, field)[0] = old[0] + 64
    with pytest.raises(ValueError):
        call(p, **calls[name])
    getattr(p, field)[0] = old[0]
    with pytest.raises(Called):
        call(p, **calls[name])


def test_strided_tensors_with_their_own_parameters_pass():
    _, calls = _paged()
    wide = torch.zeros(6, 12, 64, dtype=BF)
    pools = torch.zeros(5, 2, 16, 2, 64, dtype=BF)                       # K and V of a page side by side
    Q, O, K, V = wide[:, 0:4], wide[:, 4:8], wide[:, 8:10], wide[:, 10:12]
    Kp, Vp = pools[:, 0], pools[:, 1]
    p = B.params_for_paged(Kp, Vp, calls["append"]["page_table"], h_q=4, Q=Q, O=O, K=K, V=V)
    for name, more in (("append", dict(Q=Q, Qout=O, K=K, V=V, Vpool=Vp)), ("attend_chunk", dict(Q=Q, O=O, Vpool=Vp)), ("key_mass", dict(Q=Q)),
                       ("evict", dict(Vpool=Vp, Kdst=torch.zeros_like(pools)[:, 0], Vdst=torch.zeros_like(pools)[:, 1]))):
        with pytest.raises(Called):
            getattr(B, f"dash_attn_{name}_paged")(p, **{**calls[name], "Kpool": Kp, **more})


@pytest.mark.parametrize("sizes", [dict(rows=1), dict(h_kv=1, h_q=1), dict(rows=1, h_kv=1, h_q=4, pages=1), dict(rows=0)])
def test_strides_of_dimensions_of_one_do_not_matter(sizes):
    p, calls = _paged(**sizes)

    def restride(t):
        return t.as_strided(t.shape, [s if n > 1 else 8 * (s + 3) for s, n in zip(t.stride(), t.shape)]) if t.numel() else t
    for name, args in LAYOUTS.items():
        kw = dict(calls[name])
        for arg in args:
            kw[arg] = restride(kw[arg])
        with pytest.raises(Called):
            getattr(B, f"dash_attn_{name}_paged")(p, **kw)


@pytest.mark.parametrize("name", ["attend_chunk", "key_mass"])
def test_workspaces_elsewhere_or_repeated_are_refused(name):
    p, calls = _paged()
    call = getattr(B, f"dash_attn_{name}_paged")
    far = torch.zeros(1 << 20, dtype=torch.uint8).as_subclass(Far)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 26), torch.zeros(64, dtype=torch.uint8)[::2], far):
        with pytest.raises(ValueError):
            call(p, **{**calls[name], "workspace": ws})


def test_rope_layouts():
    x, k = torch.zeros(2, 8, 4, 64, dtype=BF), torch.zeros(2, 8, 2, 64, dtype=BF)
    pos, rope = torch.zeros(1, 2, 8, dtype=I32), B.make_rope([1.0] * 32)
    p = B.make_params(batch=2, seq_q=8, seq_kv=8, h_q=4, h_kv=2, head_dim=64, block=64, dtype=BF, alpha=1.5)
    wide = torch.zeros(2, 8, 8, 64, dtype=BF)
    with pytest.raises(Called):
        B.dash_attn_rope(p, rope, pos, x, k, x, k)
    # both of a stride that the parameters do not have; one side only; the parameters of a wider tensor
    for q, out in ((wide[:, :, :4], wide[:, :, 4:]), (x, wide[:, :, :4]), (wide[:, :, :4], x), (x.transpose(0, 1).contiguous().transpose(0, 1),) * 2):
        with pytest.raises(ValueError):
            B.dash_attn_rope(p, rope, pos, q, None, out, None)
    fused = B.make_params(batch=2, seq_q=8, seq_kv=8, h_q=4, h_kv=2, head_dim=64, block=64, dtype=BF, alpha=1.5, q_stride=wide.stride()[:3])
    with pytest.raises(ValueError):
        B.dash_attn_rope(fused, rope, pos, x, None, x, None)
    with pytest.raises(Called):
        B.dash_attn_rope(fused, rope, pos, wide[:, :, :4], k, wide[:, :, 4:], k)
    fused.q_stride[1] = 256
    with pytest.raises(ValueError):
        B.dash_attn_rope(fused, rope, pos, wide[:, :, :4], None, wide[:, :, 4:], None)
    kv = torch.zeros(2, 8, 2, 2, 64, dtype=BF)
    with pytest.raises(ValueError):
        B.dash_attn_rope(p, rope, pos, None, kv[:, :, 0], None, kv[:, :, 1])
    with pytest.raises(ValueError):
        B.dash_attn_rope(p, rope, pos, None, k[..., ::2].repeat(1, 1, 1, 2)[..., ::2], None, k)


def test_parameters_may_be_copied():
    p, calls = _paged()
    with pytest.raises(Called):
        B.dash_attn_attend_chunk_paged(p, **calls["attend_chunk"])
    q = B.DashPagedParams()
    ctypes.memmove(ctypes.byref(q), ctypes.byref(p), ctypes.sizeof(p))
    q.h_q = 2
    with pytest.raises(ValueError):
        B.dash_attn_attend_chunk_paged(q, **calls["attend_chunk"])


@pytest.mark.parametrize("kw", [dict(sinks=1 << 32), dict(recent=1 << 32), dict(sinks=-(1 << 32)), dict(sinks=(1 << 32) + 1, recent=-(1 << 32))])
def test_counts_beyond_32_bits_are_not_cut_down(kw):
    """ctypes keeps the low 32 bits of what it is given: 2^32 sinks would have been none."""
    p, calls = _paged()
    with pytest.raises(ValueError):
        B.dash_attn_evict_paged(p, **{**calls["evict"], **kw})
