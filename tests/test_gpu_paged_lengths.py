"""The operators around the paged cache at lengths out of range, over shared pages and in captured graphs, where the other tests are
coarse or do not go (tolerances: test_gpu_paged_operators.py)."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2605_18753_b200 import binding as B
from tests.test_gpu_paged_operators import BF, DEV, F32, Cache, half_step, np64

pytestmark = pytest.mark.gpu


def _check(c, b, rows, K, V, q_len, kv):
    """O and lse of `rows` against the definition over the slots that exist."""
    r = half_step(BF) if c.dtype == BF else 2.0 ** -22
    Q = np64(c.Q[rows])
    ref, ref_lse, absv = po.chunk_attention(Q, K, V, q_len, kv)
    es = c.score_noise(b, Q)
    tol = (r + 2 * es + 2.0 ** -19) * absv + r * np.abs(ref) + 1e-30
    err = np.abs(np64(c.O[rows]) - ref)
    assert (err <= tol).all(), float((err / tol).max())
    got = np64(c.lse[rows])
    assert np.isfinite(ref_lse).all() and (np.abs(got - ref_lse) <= es + 2.0 ** -20 * (1 + np.abs(ref_lse))).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,page,width", [(64, 32, 2), (128, 48, 9)])
def test_lengths_beyond_the_table_see_every_slot_once(dtype, d, page, width):
    """kv_len beyond the table (rows at slots that do not exist see all that do) and negative, q_start beyond the rows."""
    n = page * width
    c = Cache([2, 2], [n, 64], h_q=4, h_kv=2, d=d, page=page, dtype=dtype, tail=1, width=width)
    c.kv_len.copy_(torch.tensor([n + 1000, -5]))
    c.q_start.copy_(torch.tensor([0, 2, 50]))
    c.attend()
    _check(c, 0, slice(0, 2), np64(c.Kc[0]), np64(c.Vc[0]), 2, n + 1000)
    assert (c.O[2:] == 0).all() and torch.isneginf(c.lse[2:]).all()
    # the last slots just inside, at the end, and just out
    for kv in (n - 1, n, n + 1, (1 << 31) - 1):
        c.kv_len.copy_(torch.tensor([kv, 3]))
        c.q_start.copy_(torch.tensor([0, 2, 4]))
        c.O.fill_(7.0), c.lse.fill_(7.0)
        c.attend()
        have = min(kv, n)
        _check(c, 0, slice(0, 2), np64(c.Kc[0])[:have], np64(c.Vc[0])[:have], 2, kv)
        _check(c, 1, slice(2, 4), np64(c.Kc[1])[:3], np64(c.Vc[1])[:3], 2, 3)
        assert (c.O[4:] == 7).all() and (c.lse[4:] == 7).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_sequences_that_share_pages(dtype):
    """A common prefix is one set of pages in several tables, and a page may stand in a table twice."""
    c = Cache([1, 30, 1], [640, 640, 640], h_q=8, h_kv=2, d=128, page=64, dtype=dtype)
    c.table[1, :6] = c.table[0, :6]
    c.table[2, :6] = c.table[0, :6]
    c.table[2, 7] = c.table[2, 6]
    for b in (1, 2):
        slot = torch.arange(640, device=DEV)
        c.Kc[b], c.Vc[b] = (t[c.table[b, slot // 64].long(), slot % 64].cpu() for t in (c.Kpool, c.Vpool))
    c.attend()
    c.check_attention()
    out = torch.full((3, 2, c.cap), 9.0, device=DEV)
    B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, None, out, c.ws)
    c.check_mass(None, 1.0, out)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_whole_step_in_a_graph(dtype):
    """Append, attention, weights and eviction in place, captured once, replayed for other lengths, tokens and positions: the same bits
    as the calls one by one."""
    b, h_q, h_kv, d, page, width, keep = 3, 8, 2, 128, 64, 6, 200
    g = torch.Generator().manual_seed(5)
    table = torch.randperm(b * width, generator=g).view(b, width).to(torch.int32).to(DEV)
    rope = B.make_rope([10000.0 ** (-i / 64) for i in range(64)], axis=[i % 2 for i in range(64)])
    Kp, Vp = (torch.zeros(b * width, page, h_kv, d, dtype=dtype, device=DEV) for _ in range(2))
    Q, K, V = (torch.zeros(5, h, d, dtype=dtype, device=DEV) for h in (h_q, h_kv, h_kv))
    Qr, O, lse = torch.zeros_like(Q), torch.zeros_like(Q), torch.zeros(5, h_q, device=DEV)
    pos, mass = torch.zeros(2, 5, dtype=torch.int32, device=DEV), torch.zeros(b, h_kv, width * page, device=DEV)
    q_start, kv_len, new_len = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (b + 1, b, b))
    kept = torch.zeros(b, h_kv, keep, dtype=torch.int32, device=DEV)
    p = B.params_for_paged(Kp, Vp, table, h_q=h_q, Q=Q, O=O, K=K, V=V)
    ws = B.alloc_paged_workspace(p)
    state = (Kp, Vp, Qr, O, lse, mass, kept, new_len)

    def step():
        B.dash_attn_append_paged(p, rope, pos, q_start, kv_len, table, Q, Qr, K, V, Kp, Vp)
        B.dash_attn_attend_chunk_paged(p, Qr, Kp, Vp, table, q_start, kv_len, O, lse, ws)
        B.dash_attn_key_mass_paged(p, Qr, Kp, table, q_start, kv_len, lse, mass, mass, ws, decay=0.9)
        B.dash_attn_evict_paged(p, mass, kv_len, table, Kp, Vp, kept, new_len, table, Kp, Vp, mass, keep=keep, sinks=2, recent=20)

    step()                                   # (nothing cached, no rows: loads the kernels)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k, (new, kv) in enumerate((([1, 3, 1], [50, 300, 384]), ([5, 0, 0], [384, 10, 201]), ([1, 1, 1], [200, 201, 199]))):
        for t in (Q, K, V, Kp, Vp):
            t.copy_(torch.randn(t.shape, generator=g))
        mass.copy_(torch.rand(mass.shape, generator=g))
        pos.copy_(torch.randint(0, 5000, pos.shape, generator=g))
        q_start.copy_(torch.tensor([0] + [sum(new[:i + 1]) for i in range(b)]))
        kv_len.copy_(torch.tensor(kv))
        before = [t.clone() for t in state]
        graph.replay()
        torch.cuda.synchronize()
        assert B.dash_attn_last_status(ws) == 0
        replayed = [t.clone() for t in state]
        for t, old in zip(state, before):
            t.copy_(old)
        step()
        assert all(torch.equal(x, y) for x, y in zip(replayed, state)), k
        assert new_len.tolist() == [min(n, keep) for n in kv]


def test_evictions_on_two_streams():
    """Caches of their own, moved at the same time (no workspace is shared: there is none)."""
    def make(seed):
        c = Cache([0, 0], [3000, 500 + seed], h_q=4, h_kv=2, d=64, page=64, dtype=BF, seed=seed)
        mass = torch.rand(2, 2, c.cap, generator=torch.Generator().manual_seed(seed)).to(DEV)
        return c, mass, torch.empty(2, 2, 400, dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    sets = [make(k) for k in range(2)]
    old = [(c.Kpool.clone(), c.Vpool.clone(), m.clone()) for c, m, _, _ in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for (c, mass, kept, new_len), s in zip(sets, streams):
        with torch.cuda.stream(s):
            B.dash_attn_evict_paged(c.p, mass, c.kv_len, c.table, c.Kpool, c.Vpool, kept, new_len, c.table, c.Kpool, c.Vpool, mass, keep=400,
                                    sinks=3, recent=50)
    torch.cuda.synchronize()
    for (c, mass, kept, new_len), (K, V, m) in zip(sets, old):
        for b, n in enumerate(c.kv_lens):
            for r in range(2):
                want = po.evicted(np64(m[b, r]), n, 400, 3, 50)
                src, j = torch.from_numpy(want).to(DEV), torch.arange(len(want), device=DEV)
                assert kept[b, r, :len(want)].tolist() == want.tolist()
                for now, then in ((c.Kpool, K), (c.Vpool, V)):
                    assert torch.equal(now[c.table[b, j // 64].long(), j % 64, r], then[c.table[b, src // 64].long(), src % 64, r])
