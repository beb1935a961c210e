"""The operators around the paged cache (rotary positions, append, chunk attention, key mass, eviction) against their float64
definitions, at the lengths, layouts and contents where they can go wrong.

Tolerances, from the roundings that the operators document:
* rotation: cosine and sine within 3e-7, two products and a sum in fp32 -> 6e-7 (|x| + |y|); a bf16 output adds half a step, 2^-8.
* scores: fp32 sums of d products, in any order and with truncation: es = d 2^-23 max_t sum |q k_t| / sqrt(d).  A weight is then off by
  at most (es + 2^-20) of itself, lse by es + 2^-20 (1 + |lse|).
* attention: weights (bf16: rounded, 2^-8 of each) times |v|, and the division by their unrounded sum, so |O - O*| <=
  (r + 2 es + 2^-19) sum p|v| + r |O| with r = 2^-8 for bf16 and 2^-22 for fp32.
* mass: the weights' error, times the row sums' fp32 noise 2^-20."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2605_18753_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def np64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def half_step(dtype):
    return 2.0 ** -8 if dtype == BF else 2.0 ** -24


class Cache:
    """Paged caches of several sequences with their packed new rows.  Slots behind kv_len, unused pages and rows that belong to no
    sequence hold NaN."""

    def __init__(self, q_lens, kv_lens, *, h_q, h_kv, d, page, dtype, seed=0, lead=0, tail=0, spare=2, width=None, q_scale=2.0):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.q_lens, self.kv_lens, self.h_q, self.h_kv, self.d, self.page, self.dtype = q_lens, kv_lens, h_q, h_kv, d, page, dtype
        need = [-(-n // page) for n in kv_lens]
        self.width = width or max(max(need), 1)
        total = sum(need) + spare
        order = torch.randperm(total, generator=g).to(torch.int32)
        self.table = torch.full((len(q_lens), self.width), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.q_start = torch.tensor([lead] + [lead + sum(q_lens[:b + 1]) for b in range(len(q_lens))], dtype=torch.int32)
        self.rows = lead + sum(q_lens) + tail
        nan = float("nan")
        self.Kc = [rnd(n, h_kv, d).to(dtype) for n in kv_lens]
        self.Vc = [rnd(n, h_kv, d).to(dtype) for n in kv_lens]
        self.Kpool, self.Vpool = (torch.full((total, page, h_kv, d), nan, dtype=dtype) for _ in range(2))
        for b, n in enumerate(kv_lens):
            for p in range(need[b]):
                m = min(page, n - p * page)
                self.Kpool[self.table[b, p], :m] = self.Kc[b][p * page:p * page + m]
                self.Vpool[self.table[b, p], :m] = self.Vc[b][p * page:p * page + m]
        self.Q = torch.full((self.rows, h_q, d), nan, dtype=dtype)
        self.Q[lead:lead + sum(q_lens)] = (rnd(sum(q_lens), h_q, d) * q_scale).to(dtype)
        for name in ("table", "q_start", "Kpool", "Vpool", "Q"):
            setattr(self, name, getattr(self, name).to(DEV))
        self.kv_len = torch.tensor(kv_lens, dtype=torch.int32, device=DEV)
        self.O = torch.full_like(self.Q, 7.0)
        self.lse = torch.full((self.rows, h_q), 7.0, device=DEV)
        self.p = B.params_for_paged(self.Kpool, self.Vpool, self.table, h_q=h_q, Q=self.Q, O=self.O)
        self.ws = B.alloc_paged_workspace(self.p)

    @property
    def cap(self):
        return self.width * self.page

    def spans(self):
        s = self.q_start.tolist()
        return [(b, s[b], s[b + 1]) for b in range(len(self.q_lens))]

    def attend(self, O=None, lse="own"):
        lse = self.lse if isinstance(lse, str) else lse
        B.dash_attn_attend_chunk_paged(self.p, self.Q, self.Kpool, self.Vpool, self.table, self.q_start, self.kv_len,
                                       self.O if O is None else O, lse, self.ws)
        assert B.dash_attn_last_status(self.ws) == 0

    def score_noise(self, b, q):
        """es of the sequence (top of the file)."""
        g = self.h_q // self.h_kv
        k = np.abs(np64(self.Kc[b]))
        if not len(k) or not len(q):
            return 0.0
        return self.d * 2.0 ** -23 * max(float((np.abs(q[:, h]) @ k[:, h // g].T).max()) for h in range(self.h_q)) / np.sqrt(self.d)

    def check_attention(self):
        r = half_step(self.dtype) if self.dtype == BF else 2.0 ** -22
        O, lse, Q = np64(self.O), np64(self.lse), np64(self.Q)
        for b, a, e in self.spans():
            ref, ref_lse, absv = po.chunk_attention(Q[a:e], np64(self.Kc[b]), np64(self.Vc[b]), e - a, self.kv_lens[b])
            es = self.score_noise(b, Q[a:e])
            tol = (r + 2 * es + 2.0 ** -19) * absv + r * np.abs(ref) + 1e-30
            assert np.isfinite(O[a:e]).all()
            assert (np.abs(O[a:e] - ref) <= tol).all(), (b, float((np.abs(O[a:e] - ref) / tol).max()))
            none = np.isneginf(ref_lse)
            assert np.array_equal(none, np.isneginf(lse[a:e])) and (O[a:e][none] == 0).all()
            err = np.abs(np.where(none, 0, lse[a:e]) - np.where(none, 0, ref_lse))
            assert (err <= es + 2.0 ** -20 * (1 + np.abs(np.where(none, 0, ref_lse)))).all(), (b, err.max())
        out = np.ones(self.rows, dtype=bool)
        out[self.q_start[0].item():self.q_start[-1].item()] = False
        assert (O[out] == 7).all() and (lse[out] == 7).all()        # rows of no sequence: as they were

    def check_mass(self, mass_in, decay, got):
        Q, lse = np64(self.Q), np64(self.lse)
        for b, a, e in self.spans():
            n = self.kv_lens[b]
            old = None if mass_in is None else np64(mass_in[b, :, :n])
            ref = po.key_mass(Q[a:e], np64(self.Kc[b]), lse[a:e], e - a, n, old, decay)
            es = self.score_noise(b, Q[a:e])
            tol = (es + 2.0 ** -20 * (1 + np.abs(lse[a:e][np.isfinite(lse[a:e])]).max(initial=0.0)) + 2.0 ** -19) * np.abs(ref) + 1e-30
            err = np.abs(np64(got[b, :, :n]) - ref)
            assert (err <= tol).all(), (b, float((err / tol).max()))
            assert (got[b, :, n:] == 9).all()                       # slots behind the cache: as they were


SHAPES = [
    # (q_lens, kv_lens, h_q, h_kv, d, page, dtype)
    ([1], [1], 4, 1, 128, 64, BF),
    ([1, 1, 1], [128, 129, 127], 8, 2, 128, 64, BF),
    ([1, 3, 0, 17], [500, 3, 40, 300], 32, 8, 128, 16, BF),
    ([200], [200], 8, 2, 64, 48, BF),
    ([300, 1, 70], [777, 900, 70], 12, 4, 64, 80, BF),                # three heads a group: 126 of 128 rows
    ([65, 64, 63], [65, 640, 191], 16, 4, 128, 128, BF),
    ([130], [1030], 2, 2, 128, 256, BF),                              # one head a group
    ([33, 2], [400, 260], 16, 1, 64, 32, BF),                         # sixteen heads a group
    ([5], [130], 71, 1, 64, 16, BF),                                  # one token a tile
    ([2, 1], [140, 33], 128, 1, 128, 64, BF),
    ([6, 2], [3, 1], 8, 2, 128, 16, BF),                              # more rows than slots: some see nothing
    ([1] * 40, [1 + 7 * k for k in range(40)], 4, 2, 64, 16, BF),
    ([1], [1], 2, 2, 64, 16, F32),
    ([1, 30, 0], [333, 64, 10], 8, 2, 128, 48, F32),
    ([70, 5], [129, 300], 6, 2, 64, 16, F32),
    ([100], [100], 4, 4, 128, 64, F32),
    ([4, 3], [2, 20], 10, 1, 64, 32, F32),
]


@pytest.mark.parametrize("q_lens,kv_lens,h_q,h_kv,d,page,dtype", SHAPES)
def test_chunk_attention(q_lens, kv_lens, h_q, h_kv, d, page, dtype):
    c = Cache(q_lens, kv_lens, h_q=h_q, h_kv=h_kv, d=d, page=page, dtype=dtype, lead=2, tail=3)
    c.attend()
    c.check_attention()
    first, lse = c.O.clone(), c.lse.clone()
    c.O.fill_(7.0)
    c.attend(lse=None)                             # without lse, and a second time on the workspace
    assert torch.equal(c.O, first) and torch.equal(c.lse, lse)


@pytest.mark.parametrize("q_lens,kv_lens,h_q,h_kv,d,page,dtype", SHAPES)
def test_key_mass(q_lens, kv_lens, h_q, h_kv, d, page, dtype):
    c = Cache(q_lens, kv_lens, h_q=h_q, h_kv=h_kv, d=d, page=page, dtype=dtype, lead=1, tail=2)
    c.attend()
    mass_in = torch.rand(len(q_lens), h_kv, c.cap, device=DEV)
    for b, n in enumerate(kv_lens):
        mass_in[b, :, max(0, n - q_lens[b]):] = float("nan")          # new slots and those behind: never read
    for given, decay in ((mass_in, 0.5), (None, 1.0)):
        out = torch.full((len(q_lens), h_kv, c.cap), 9.0, device=DEV)
        B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, given, out, c.ws, decay=decay)
        assert B.dash_attn_last_status(c.ws) == 0
        c.check_mass(given, decay, out)
    inplace = mass_in.clone()
    B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, inplace, inplace, c.ws, decay=0.5)
    again = torch.full_like(out, 9.0)
    B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, mass_in, again, c.ws, decay=0.5)
    for b, n in enumerate(kv_lens):
        assert torch.equal(inplace[b, :, :n], again[b, :, :n])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("q_lens,kv_lens", [([1], [9001]), ([1, 1], [5000, 130]), ([40], [6000]), ([1, 20, 1], [4097, 20, 2048])])
def test_long_caches_are_divided_among_blocks(q_lens, kv_lens, dtype):
    c = Cache(q_lens, kv_lens, h_q=4, h_kv=1, d=128, page=64, dtype=dtype, seed=5)
    c.attend()
    c.check_attention()


@pytest.mark.parametrize("length", [9 * 128 + 5, 41 * 128 + 42, 70 * 128 + 29])
def test_tail_of_the_cache_leaves_the_tiles_before_it_alone(length):
    """Rows behind the end are cleared in the last tile only: the weight of every row sits in the two tiles of 128 slots before it, in
    rows that the last tile does not have."""
    b, h_kv = 12, 8
    c = Cache([1] * b, [length] * b, h_q=16, h_kv=h_kv, d=128, page=64, dtype=BF, seed=length)
    for k in range(b):
        for tile in (2, 3):
            slot = (length // 128 + 1 - tile) * 128 + 60 + 5 * k
            c.Kc[k][slot] = 0.5 * c.Q[k].view(h_kv, 2, 128)[:, 0].cpu() + 0.5 * c.Q[k].view(h_kv, 2, 128)[:, 1].cpu()
            c.Kpool[c.table[k, slot // 64].long(), slot % 64] = c.Kc[k][slot].to(DEV)
    for _ in range(20):
        c.O.fill_(7.0)
        c.attend()
    c.check_attention()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strided_tensors(dtype):
    """Queries out of a fused projection, outputs and pools with gaps, heads before tokens in the pool."""
    c = Cache([9, 30], [100, 77], h_q=8, h_kv=2, d=64, page=32, dtype=dtype)
    wide = torch.full((c.rows, 8 + 4, 64), float("nan"), dtype=dtype, device=DEV)
    wide[:, 2:10] = c.Q
    Q, O = wide[:, 2:10], torch.full((c.rows, 10, 64), 7.0, dtype=dtype, device=DEV)[:, 1:9]
    Kp, Vp = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (c.Kpool, c.Vpool))      # [page, head, token, d] in memory
    p = B.params_for_paged(Kp, Vp, c.table, h_q=8, Q=Q, O=O)
    B.dash_attn_attend_chunk_paged(p, Q, Kp, Vp, c.table, c.q_start, c.kv_len, O, c.lse, c.ws)
    assert B.dash_attn_last_status(c.ws) == 0
    c.O.copy_(O)
    c.check_attention()


def test_pages_that_do_not_exist_read_as_zeros():
    for dtype in (BF, F32):
        c = Cache([3], [100], h_q=4, h_kv=2, d=64, page=32, dtype=dtype)
        c.table[0, 1] = -1
        c.table[0, 2] = 1 << 30
        c.Kc[0][32:96] = 0
        c.Vc[0][32:96] = 0
        c.attend()
        c.check_attention()


def test_lengths_out_of_range_leave_everything_in_place():
    """kv_len beyond the table and negative, q_start beyond the rows: clamped, nothing outside is touched."""
    for dtype in (BF, F32):
        c = Cache([2, 2], [64, 64], h_q=4, h_kv=2, d=64, page=32, dtype=dtype, tail=1)
        c.kv_len.copy_(torch.tensor([1000, -5]))
        c.q_start.copy_(torch.tensor([0, 2, 50]))
        c.attend()
        # slots 998, 999 of the first sequence see all 64 that exist; the second sequence sees nothing
        ref, _, _ = po.chunk_attention(np64(c.Q[:2]), np64(c.Kc[0]), np64(c.Vc[0]), 2, 1000)
        assert np.abs(np64(c.O[:2]) - ref).max() < 0.05
        assert (c.O[2:] == 0).all() and torch.isneginf(c.lse[2:]).all()


def test_many_sequences_take_several_launches():
    """More unit slots than one launch's plan holds."""
    n = 4500
    c = Cache([1] * n, [1 + k % 5 for k in range(n)], h_q=2, h_kv=1, d=64, page=16, dtype=BF, q_scale=1.0)
    c.attend()
    c.check_attention()
    out = torch.full((n, 1, c.cap), 9.0, device=DEV)
    B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, None, out, c.ws)
    assert B.dash_attn_last_status(c.ws) == 0
    c.check_mass(None, 1.0, out)


def test_offsets_beyond_32_bits():
    """Pools of more than 2^31 elements: the last pages are read, written and moved."""
    pages = (1 << 31) // (64 * 2 * 64) + 8
    K = torch.empty(pages, 64, 2, 64, dtype=BF, device=DEV)
    V = torch.empty_like(K)
    table = torch.tensor([[pages - 1, pages - 3]], dtype=torch.int32, device=DEV)
    K[pages - 4:].zero_(), V[pages - 4:].zero_()
    kn, vn, q = (torch.randn(100, h, 64, device=DEV).to(BF) for h in (2, 2, 4))
    q_start, kv_len = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, 100], [100]))
    O, lse = torch.empty_like(q), torch.empty(100, 4, device=DEV)
    p = B.params_for_paged(K, V, table, h_q=4, Q=q, O=O, K=kn, V=vn)
    ws = B.alloc_paged_workspace(p)
    B.dash_attn_append_paged(p, None, None, q_start, kv_len, table, None, None, kn, vn, K, V)
    assert torch.equal(K[pages - 1], kn[:64]) and torch.equal(V[pages - 3, :36], vn[64:])
    B.dash_attn_attend_chunk_paged(p, q, K, V, table, q_start, kv_len, O, lse, ws)
    assert B.dash_attn_last_status(ws) == 0
    ref, _, absv = po.chunk_attention(np64(q), np64(kn), np64(vn), 100, 100)
    assert (np.abs(np64(O) - ref) <= 2.0 ** -8 * 1.1 * (absv + np.abs(ref))).all()
    mass = torch.zeros(1, 2, 128, device=DEV)
    mass[..., 50:60] = 1
    kept, new_len = torch.empty(1, 2, 20, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
    B.dash_attn_evict_paged(p, mass, kv_len, table, K, V, kept, new_len, table, K, V, mass, keep=20, recent=10)
    want = torch.tensor(list(range(50, 60)) + list(range(90, 100)), device=DEV)
    assert (kept == want).all() and torch.equal(K[pages - 1, :20], kn[want]) and torch.equal(V[pages - 1, :20], vn[want])


def test_one_sequence_over_several_launches():
    """A sequence with more units than one launch's plan holds (two tokens a unit), behind another one."""
    c = Cache([200, 8300, 1], [200, 60, 33], h_q=128, h_kv=1, d=64, page=16, dtype=BF, q_scale=1.0)
    c.attend()
    c.check_attention()
    out = torch.full((3, 1, c.cap), 9.0, device=DEV)
    B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, None, out, c.ws)
    assert B.dash_attn_last_status(c.ws) == 0
    c.check_mass(None, 1.0, out)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("q_lens,kv_lens,h_q,h_kv", [
    ([1] * 39 + [100], [50 + k for k in range(39)] + [3000], 4, 2),      # few rows a sequence on average, one with many
    ([300], [3001], 4, 1), ([1, 200], [2500, 900], 8, 2), ([40], [9000], 2, 1)])
def test_weights_of_long_caches_are_divided_among_blocks(q_lens, kv_lens, h_q, h_kv, dtype):
    c = Cache(q_lens, kv_lens, h_q=h_q, h_kv=h_kv, d=64, page=32, dtype=dtype, seed=6)
    c.attend()
    mass = torch.rand(len(q_lens), h_kv, c.cap, device=DEV)
    out = torch.full_like(mass, 9.0)
    for _ in range(2):
        B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, mass, out, c.ws, decay=0.75)
        assert B.dash_attn_last_status(c.ws) == 0
        c.check_mass(mass, 0.75, out)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_of_minus_infinity_give_no_weight(dtype):
    """Whatever their scores are: a log-sum-exp of -inf says that the row has no weight to give."""
    c = Cache([40, 1, 3], [200, 77, 300], h_q=8, h_kv=2, d=64, page=32, dtype=dtype)
    c.attend()
    given = c.lse.clone()
    given[2], given[30, 5], given[40] = -torch.inf, -torch.inf, -torch.inf
    out = torch.full((3, 2, c.cap), 9.0, device=DEV)
    B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, given, None, out, c.ws)
    c.lse.copy_(torch.where(torch.isneginf(given), torch.inf, given))      # to the formula: weights of exp(-inf)
    c.check_mass(None, 1.0, out)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rising", [True, False])
def test_running_maximum_that_moves_with_every_tile(rising, dtype):
    """Scores that climb, or fall, by several powers of two from each tile of keys to the next."""
    c = Cache([1, 300, 7], [3000, 1500, 900], h_q=8, h_kv=2, d=128, page=64, dtype=dtype)
    u = torch.randn(128, generator=torch.Generator().manual_seed(8))
    c.Q.copy_((u * torch.linspace(0.5, 2.0, 8)[:, None]).to(dtype).to(DEV).expand_as(c.Q))
    for b, n in enumerate(c.kv_lens):
        t = torch.linspace(0, 1, n) if rising else torch.linspace(1, 0, n)
        c.Kc[b] = (u * (4 * t)[:, None, None] + 0.1 * c.Kc[b].float()).to(dtype)
        for k in range(-(-n // 64)):
            part = c.Kc[b][k * 64:k * 64 + 64]
            c.Kpool[c.table[b, k].long(), :len(part)] = part.to(DEV)
    c.attend()
    c.check_attention()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_weights_and_eviction_at_lengths_out_of_range(dtype):
    """kv_len beyond the table counts as far as there are slots, a negative one as nothing; a page that is none reads as zeros."""
    c = Cache([2, 2], [64, 64], h_q=4, h_kv=2, d=64, page=32, dtype=dtype)
    c.table[0, 1] = 1 << 29
    c.Kc[0][32:] = 0
    c.kv_len.copy_(torch.tensor([1000, -5]))
    c.attend()
    mass = torch.rand(2, 2, 64, device=DEV)
    out = torch.full_like(mass, 9.0)
    B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, mass, out, c.ws, decay=0.5)
    s = np.einsum("ihd,thd->iht", np64(c.Q[:2]), np64(c.Kc[0]).repeat(2, axis=1)) / 8
    want = 0.5 * np64(mass[0]) + np.exp(s - np64(c.lse[:2])[..., None]).sum(0).reshape(2, 2, 64).sum(1)
    es = c.score_noise(0, np64(c.Q[:2]))
    assert (np.abs(np64(out[0]) - want) <= (es + 2.0 ** -20 * (1 + np.abs(np64(c.lse[:2])).max()) + 2.0 ** -19) * want).all()
    assert (out[1] == 9).all()
    for keep in (40, 64, 70):
        kept, new_len, table, K, V, moved = _evict(c, mass, keep, 2, 5, True)
        assert new_len == [min(64, keep), 0] and (kept[1] == -1).all()
        for r in range(2):
            want = po.evicted(np64(mass[0, r]), 64, keep, 2, 5)
            assert kept[0, r, :len(want)].tolist() == want.tolist() and (kept[0, r, len(want):] == -1).all()
            assert torch.equal(moved[0, r, :len(want)], mass[0, r].cpu()[torch.from_numpy(want)])
            first = torch.from_numpy(want[:32])                      # the rows of the one page that there is
            src = c.Kpool[c.table[0, 0].long(), :, r].cpu()
            old = torch.where((first < 32)[:, None], src[first.clamp(max=31)].float(), torch.zeros(1))
            assert torch.equal(K[table[0, 0].long(), :len(first), r].float(), old)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kv", [[40, 300], [9000, 5000]])
def test_a_nan_query_stays_in_its_row(dtype, kv):
    """In whole units and in units cut among blocks."""
    c = Cache([3, 40], kv, h_q=8, h_kv=2, d=128, page=64, dtype=dtype)
    c.attend()
    O, lse = c.O.clone(), c.lse.clone()
    c.Q[1, 2, 5] = float("nan")
    c.Q[20, 7, 100] = float("nan")
    c.attend()
    hit = torch.zeros(c.rows, 8, dtype=torch.bool, device=DEV)
    hit[1, 2] = hit[20, 7] = True
    assert torch.isnan(c.O[hit]).all() and torch.isnan(c.lse[hit]).all()
    assert torch.equal(c.O[~hit], O[~hit]) and torch.equal(c.lse[~hit], lse[~hit])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("q,kv", [([3, 40], [40, 300]), ([3, 40], [9000, 5000]), ([1, 1], [9000, 64])])
def test_a_nan_key_reaches_the_rows_that_see_it(q, kv, dtype):
    c = Cache(q, kv, h_q=8, h_kv=2, d=128, page=64, dtype=dtype)
    c.attend()
    O, lse = c.O.clone(), c.lse.clone()
    slot = kv[1] - (20 if q[1] > 20 else 1)                  # in sequence 1, head 1; its last 20 tokens (or the one) see it
    c.Kpool[int(c.table[1, slot // 64]), slot % 64, 1, 7] = float("nan")
    c.attend()
    hit = torch.zeros(c.rows, 8, dtype=torch.bool, device=DEV)
    hit[q[0] + q[1] - (kv[1] - slot): q[0] + q[1], 4:] = True
    assert torch.isnan(c.O[hit]).all() and torch.isnan(c.lse[hit]).all()
    assert torch.equal(c.O[~hit], O[~hit]) and torch.equal(c.lse[~hit], lse[~hit])


def test_an_error_in_the_status_word_ends_the_call_and_stays():
    """A workspace whose status word holds an error: the blocks give up at the first wait that is not over at once, everything they have
    issued runs out, and the word keeps the first error until it is reset; then the workspace serves again."""
    c = Cache([1, 300], [4000, 900], h_q=8, h_kv=2, d=128, page=64, dtype=BF)
    mass = torch.zeros(2, 2, c.cap, device=DEV)
    for _ in range(3):
        c.ws[:4] = torch.tensor([0xf9, 0xff, 0xff, 0xff], dtype=torch.uint8)              # DASH_ERR_TIMEOUT
        B.dash_attn_attend_chunk_paged(c.p, c.Q, c.Kpool, c.Vpool, c.table, c.q_start, c.kv_len, c.O, c.lse, c.ws)
        B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, None, mass, c.ws)
        assert B.dash_attn_last_status(c.ws) == -7
    B.dash_attn_reset_status(c.ws)
    c.attend()
    c.check_attention()


# ---------------------------------------------------------------- rotary positions

def rope_tolerance(x, ref, dtype, pairs, interleaved):
    a = np.abs(x)
    swap = a.copy()
    if interleaved:
        swap[..., 0:2 * pairs:2], swap[..., 1:2 * pairs:2] = a[..., 1:2 * pairs:2], a[..., 0:2 * pairs:2]
    else:
        swap[..., :pairs], swap[..., pairs:2 * pairs] = a[..., pairs:2 * pairs], a[..., :pairs]
    return 6e-7 * (a + swap) + (half_step(dtype) * np.abs(ref) if dtype == BF else 0) + 1e-30


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,pairs,axes", [(128, 64, 3), (64, 32, 1), (64, 16, 2), (128, 20, 4), (64, 5, 2), (128, 63, 1)])
@pytest.mark.parametrize("batch,n", [(1, 1), (2, 37)])
def test_rope_forward_and_backward(dtype, interleaved, d, pairs, axes, batch, n):
    g = torch.Generator().manual_seed(pairs + n)
    h_q, h_kv = 4, 2
    Q, K = (torch.randn(batch, n, h, d, generator=g).to(dtype).to(DEV) for h in (h_q, h_kv))
    top = 1 << 31
    pos = torch.randint(-top, top, (axes, batch, n), generator=g, dtype=torch.int64).to(torch.int32).to(DEV)
    freq = [10000.0 ** (-i / pairs) for i in range(pairs)]
    axis = [i % axes for i in range(pairs)]
    rope = B.make_rope(freq, axis=axis, interleaved=interleaved)
    p = B.make_params(batch=batch, seq_q=n, seq_kv=n, h_q=h_q, h_kv=h_kv, head_dim=d, block=64, dtype=dtype, alpha=1.5)
    for inverse in (False, True):
        Qo, Ko = torch.full_like(Q, 7.0), torch.full_like(K, 7.0)
        B.dash_attn_rope(p, rope, pos, Q, K, Qo, Ko, inverse=inverse)
        for x, got in ((Q, Qo), (K, Ko)):
            flat = np64(x).reshape(batch * n, -1, d)
            ref = po.rotate(flat, pos.cpu().numpy().reshape(axes, -1), freq, axis, interleaved, inverse)
            tol = rope_tolerance(flat, ref, dtype, pairs, interleaved)
            err = np.abs(np64(got).reshape(flat.shape) - ref)
            assert (err <= tol).all(), float((err / tol).max())
            assert torch.equal(got[..., 2 * pairs:], x[..., 2 * pairs:])
        q_only, own = torch.full_like(Q, 7.0), K.clone()
        B.dash_attn_rope(p, rope, pos, Q, None, q_only, None, inverse=inverse)
        B.dash_attn_rope(p, rope, pos, None, own, None, own, inverse=inverse)      # in place
        assert torch.equal(q_only, Qo) and torch.equal(own, Ko)


def test_rope_gradient_through_a_loss():
    """The gradient of a loss of the rotated queries is the inverse rotation of its gradient there: against differences."""
    p = B.make_params(batch=1, seq_q=9, seq_kv=9, h_q=2, h_kv=2, head_dim=64, block=16, dtype=F32, alpha=1.5)
    rope = B.make_rope([0.7 ** i for i in range(32)], axis=[i % 2 for i in range(32)])
    pos = torch.arange(18, dtype=torch.int32, device=DEV).view(2, 1, 9)
    x, v = torch.randn(2, 1, 9, 2, 64, generator=torch.Generator().manual_seed(1)).to(DEV)
    out, grad = torch.empty_like(x), torch.empty_like(x)

    def loss(t):
        B.dash_attn_rope(p, rope, pos, t.contiguous(), None, out, None)
        return (out.double() ** 3).sum().item()

    base = loss(x)
    B.dash_attn_rope(p, rope, pos, (3 * out ** 2).contiguous(), None, grad, None, inverse=True)
    eps = 1e-2
    slope = (loss(x + eps * v) - loss(x - eps * v)) / (2 * eps)
    # a cubic: the central difference is off by eps^2 sum (R v)^3; fp32 forwards leave 1e-6 of the sum of |terms| over 2 eps
    noise = 1e-6 * (x.abs().double() ** 3).sum().item() * 8 / eps + eps ** 2 * (v.abs().double() ** 3).sum().item() * 3
    assert abs(slope - (grad.double() * v.double()).sum().item()) <= noise and np.isfinite(base)


def test_rope_strided_batches():
    p_shape = dict(batch=2, seq_q=50, seq_kv=50, h_q=4, h_kv=2, head_dim=64, block=64, dtype=BF, alpha=1.5)
    qkv = torch.randn(2, 50, 8, 64, device=DEV).to(BF)
    Q, K = qkv[:, :, :4], qkv[:, :, 4:6]
    p = B.make_params(**p_shape, q_stride=B._strides3(Q), k_stride=B._strides3(K))
    rope = B.make_rope([0.5 ** i for i in range(32)])
    pos = torch.arange(100, dtype=torch.int32, device=DEV).view(1, 2, 50)
    ref_q, ref_k = torch.empty(2, 50, 4, 64, dtype=BF, device=DEV), torch.empty(2, 50, 2, 64, dtype=BF, device=DEV)
    B.dash_attn_rope(B.make_params(**p_shape), rope, pos, Q.contiguous(), K.contiguous(), ref_q, ref_k)
    v = qkv[:, :, 6:].clone()
    B.dash_attn_rope(p, rope, pos, Q, K, Q, K)                        # in place inside the fused tensor
    assert torch.equal(Q, ref_q) and torch.equal(K, ref_k) and torch.equal(qkv[:, :, 6:], v)


# ---------------------------------------------------------------- append

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("q_lens,kv_lens,page,pairs,interleaved", [
    ([1, 1, 1], [1, 64, 65], 64, 64, False), ([5, 0, 40], [9, 3, 40], 16, 16, True), ([3, 2], [2, 900], 48, 7, False),
    ([700, 900], [700, 1000], 128, 64, False), ([2, 4], [40, 7], 32, 0, False)])
def test_append(dtype, q_lens, kv_lens, page, pairs, interleaved):
    h_q, h_kv, d, axes = 6, 2, 128, 2
    c = Cache(q_lens, [min(n, 200) for n in kv_lens], h_q=h_q, h_kv=h_kv, d=d, page=page, dtype=dtype, lead=1, tail=2,
              width=-(-200 // page) if max(kv_lens) == 900 else -(-max(kv_lens) // page), spare=40)
    # every sequence gets pages of its own for all of its slots; one entry is no page
    pages = c.Kpool.shape[0]
    need = c.table.numel()
    if need > pages:
        c.Kpool, c.Vpool = (torch.full((need, page, h_kv, d), 5.0, dtype=dtype, device=DEV) for _ in range(2))
        pages = need
    c.Kpool.fill_(5.0), c.Vpool.fill_(5.0)
    c.table.copy_(torch.randperm(pages, generator=torch.Generator().manual_seed(3))[:need].view_as(c.table))
    c.table[-1, -1] = -1
    c.kv_len.copy_(torch.tensor(kv_lens))
    g = torch.Generator().manual_seed(4)
    K, V = (torch.randn(c.rows, h_kv, d, generator=g).to(dtype).to(DEV) for _ in range(2))
    pos = torch.randint(0, 100000, (axes, c.rows), generator=g).to(torch.int32).to(DEV)
    freq, axis = [10000.0 ** (-i / max(pairs, 1)) for i in range(pairs)], [i % axes for i in range(pairs)]
    rope = B.make_rope(freq, axis=axis, interleaved=interleaved) if pairs else None
    if pairs:
        pos = pos[:rope.axes].contiguous()
    p = B.params_for_paged(c.Kpool, c.Vpool, c.table, h_q=h_q, Q=c.Q, O=c.O, K=K, V=V)
    B.dash_attn_append_paged(p, rope, pos if pairs else None, c.q_start, c.kv_len, c.table, c.Q, c.O, K, V, c.Kpool, c.Vpool)
    turned = lambda x: po.rotate(np64(x), pos.cpu().numpy(), freq, axis, interleaved) if pairs else np64(x)  # noqa: E731
    want_k, want_v = (np.full(c.Kpool.shape, 5.0) for _ in range(2))
    tol_k, tk = np.zeros(c.Kpool.shape), turned(K)
    tol = rope_tolerance(np64(K), tk, dtype, pairs, interleaved) if pairs else np.zeros(tk.shape)
    inside = np.zeros(c.rows, dtype=bool)
    for b, a, e in c.spans():
        inside[a:e] = True
        for i, slot in enumerate(po.slots(e - a, kv_lens[b])):
            if 0 <= slot < c.cap and c.table[b, slot // page] >= 0:
                at = (int(c.table[b, slot // page]), slot % page)
                want_k[at], tol_k[at], want_v[at] = tk[a + i], tol[a + i], np64(V[a + i])
    assert (np.abs(np64(c.Kpool) - want_k) <= tol_k).all() and np.array_equal(np64(c.Vpool), want_v)
    tq = turned(c.Q)
    tol_q = rope_tolerance(np64(c.Q), tq, dtype, pairs, interleaved) if pairs else np.zeros(tq.shape)
    assert (np.abs(np64(c.O) - tq)[inside] <= tol_q[inside]).all() and (c.O[~torch.from_numpy(inside)] == 7).all()


# ---------------------------------------------------------------- eviction

def _evict(c, mass, keep, sinks, recent, in_place):
    b = len(c.kv_lens)
    kept = torch.full((b, c.h_kv, keep), -9, dtype=torch.int32, device=DEV)
    new_len = torch.full((b,), -9, dtype=torch.int32, device=DEV)
    if in_place:
        table, K, V, out = c.table, c.Kpool.clone(), c.Vpool.clone(), mass.clone()
        B.dash_attn_evict_paged(c.p, out, c.kv_len, table, K, V, kept, new_len, table, K, V, out, keep=keep, sinks=sinks, recent=recent)
    else:
        width = -(-min(keep, c.cap) // c.page)
        K, V = (torch.full((b * width + 1, c.page, c.h_kv, c.d), 5.0, dtype=c.dtype, device=DEV) for _ in range(2))
        table = torch.randperm(b * width + 1, generator=torch.Generator().manual_seed(2))[: b * width].view(b, width).to(torch.int32).to(DEV)
        out = torch.full((b, c.h_kv, width * c.page), 5.0, device=DEV)
        B.dash_attn_evict_paged(c.p, mass, c.kv_len, c.table, c.Kpool, c.Vpool, kept, new_len, table, K, V, out, keep=keep, sinks=sinks,
                                recent=recent)
    return kept.cpu().numpy(), new_len.tolist(), table.cpu(), K.cpu(), V.cpu(), out.cpu()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kv_lens,page,keep,sinks,recent,kind", [
    ([1, 5, 40], 16, 8, 1, 2, "random"), ([300, 299, 17], 48, 33, 4, 29, "ties"), ([700, 64, 513], 64, 256, 4, 32, "zeros"),
    ([200], 32, 1, 0, 0, "random"), ([200, 0], 16, 199, 0, 0, "special"), ([90, 90], 16, 90, 3, 5, "random"), ([50], 16, 4000, 3, 5, "random"),
    ([5000, 9000], 64, 1000, 4, 64, "ties"), ([20000], 128, 777, 0, 0, "random")])
def test_evict(dtype, kv_lens, page, keep, sinks, recent, kind):
    c = Cache([0] * len(kv_lens), kv_lens, h_q=4, h_kv=2, d=64, page=page, dtype=dtype, seed=len(kv_lens))
    g = torch.Generator().manual_seed(keep)
    mass = torch.randn(len(kv_lens), 2, c.cap, generator=g).exp()
    if kind == "ties":
        mass = (mass * 2).round()
    elif kind == "zeros":
        mass = torch.where(mass < 1.5, torch.zeros_like(mass), mass)
        mass[:, :, ::7] = -0.0
    elif kind == "special":
        mass = torch.randn(len(kv_lens), 2, c.cap, generator=g)
        mass[:, :, 3::11], mass[:, :, 5::13], mass[:, :, 7::17] = float("nan"), float("inf"), float("-inf")
    mass = mass.to(DEV)
    for in_place in (False, True):
        kept, new_len, table, K, V, out = _evict(c, mass, keep, sinks, recent, in_place)
        before = {"K": c.Kpool.cpu(), "V": c.Vpool.cpu(), "mass": mass.cpu()}
        for b, n in enumerate(kv_lens):
            assert new_len[b] == min(n, keep)
            for r in range(2):
                want = po.evicted(np64(mass[b, r]), n, keep, sinks, recent)
                assert kept[b, r, :len(want)].tolist() == want.tolist() and (kept[b, r, len(want):] == -1).all()
                j = torch.arange(len(want))
                src = torch.from_numpy(want)
                for name, got in (("K", K), ("V", V)):
                    rows = got[table[b, j // page].long(), j % page, r]
                    assert torch.equal(rows, before[name][c.table.cpu()[b, src // page].long(), src % page, r])
                assert torch.equal(out[b, r, :len(want)].nan_to_num(-3.0), before["mass"][b, r, src].nan_to_num(-3.0))
                # slots behind the new length: as they were
                j = torch.arange(len(want), table.shape[1] * page)
                there = table[b, j // page] >= 0
                rest = K[table[b, j // page].long().clamp(min=0), j % page, r][there]
                if in_place:
                    old = before["K"][table[b, j // page].long().clamp(min=0), j % page, r][there]
                    assert torch.equal(rest.nan_to_num(3.0), old.nan_to_num(3.0))
                    assert torch.equal(out[b, r, len(want):].nan_to_num(3.0), before["mass"][b, r, len(want):].nan_to_num(3.0))
                else:
                    assert (rest == 5).all() and (out[b, r, len(want):] == 5).all()


def test_evict_more_slots_than_shared_memory_holds():
    """A table wide enough that a block's share of the mass does not fit on chip: the keys are read again every pass."""
    n, page, keep = 400000, 256, 1000
    width = -(-n // page)
    K = torch.randn(width, page, 1, 64, device=DEV).to(BF)
    table = torch.randperm(width, device=DEV).to(torch.int32).view(1, -1)
    mass = (torch.rand(1, 1, width * page, device=DEV) * 50000).round()
    kv_len = torch.tensor([n], dtype=torch.int32, device=DEV)
    to = torch.arange(4, dtype=torch.int32, device=DEV).view(1, 4)
    Kd, Vd = torch.zeros(4, page, 1, 64, dtype=BF, device=DEV), torch.zeros(4, page, 1, 64, dtype=BF, device=DEV)
    kept, new_len = torch.empty(1, 1, keep, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
    p = B.params_for_paged(K, K, table, h_q=1, rows=0)
    B.dash_attn_evict_paged(p, mass, kv_len, table, K, K, kept, new_len, to, Kd, Vd, keep=keep, sinks=2, recent=10)
    want = po.evicted(np64(mass[0, 0]), n, keep, 2, 10)
    assert kept[0, 0].tolist() == want.tolist() and new_len.item() == keep
    src = torch.from_numpy(want).to(DEV)
    assert torch.equal(Kd.view(-1, 64)[:keep], K[table[0, src // page].long(), src % page, 0])


# ---------------------------------------------------------------- together, in streams and graphs

def test_serving_run_together():
    """A prompt in two chunks, the routed decode over the same pages, weights, eviction, and on: every step against the float64
    definitions of what the cache then holds."""
    b, h_q, h_kv, d, page, width = 2, 8, 2, 128, 64, 8
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    g = torch.Generator().manual_seed(8)
    table = torch.randperm(b * width, generator=g).view(b, width).to(torch.int32).to(DEV)
    Kp, Vp = (torch.full((b * width, page, h_kv, d), float("nan"), dtype=BF, device=DEV) for _ in range(2))
    rope = B.make_rope([10000.0 ** (-i / 64) for i in range(64)], axis=[i * 3 // 64 for i in range(64)])
    mass = torch.zeros(b, h_kv, width * page, device=DEV)
    lens = [0, 0]
    for step, new in enumerate(([200, 130], [57, 250], [1, 1])):
        rows = sum(new)
        lens = [x + n for x, n in zip(lens, new)]
        Q, K, V = (torch.randn(rows, h, d, generator=g).to(BF).to(DEV) for h in (h_q, h_kv, h_kv))
        pos = torch.randint(0, 500, (3, rows), generator=g).to(torch.int32).to(DEV)
        O, lse = torch.empty_like(Q), torch.empty(rows, h_q, device=DEV)
        p = B.params_for_paged(Kp, Vp, table, h_q=h_q, Q=Q, O=O, K=K, V=V)
        ws = B.alloc_paged_workspace(p)
        q_start, kv_len = dev([0, new[0], rows]), dev(lens)
        B.dash_attn_append_paged(p, rope, pos, q_start, kv_len, table, Q, Q, K, V, Kp, Vp)
        B.dash_attn_attend_chunk_paged(p, Q, Kp, Vp, table, q_start, kv_len, O, lse, ws)
        B.dash_attn_key_mass_paged(p, Q, Kp, table, q_start, kv_len, lse, mass, mass, ws, decay=0.9)
        assert B.dash_attn_last_status(ws) == 0
        for s in range(b):
            slot = torch.arange(lens[s], device=DEV)
            k, v = (t[table[s, slot // page].long(), slot % page] for t in (Kp, Vp))
            a, e = q_start[s].item(), q_start[s + 1].item()
            ref, ref_lse, absv = po.chunk_attention(np64(Q[a:e]), np64(k), np64(v), e - a, lens[s])
            assert (np.abs(np64(O[a:e]) - ref) <= 2.0 ** -8 * 1.1 * (absv + np.abs(ref)) + 1e-6).all(), step
            assert np.abs(np64(lse[a:e]) - ref_lse).max() < 1e-4
        if step == 1:
            total = mass.sum().item()
            # weights of a row add up to one: 330 rows decayed once, 307 new ones, h_q heads each
            assert abs(total - h_q * (0.9 * 330 + 307)) < 1e-3 * total
            kept, new_len = torch.empty(b, h_kv, 128, dtype=torch.int32, device=DEV), torch.empty(b, dtype=torch.int32, device=DEV)
            B.dash_attn_evict_paged(p, mass, kv_len, table, Kp, Vp, kept, new_len, table, Kp, Vp, mass, keep=128, sinks=4, recent=32)
            lens = new_len.tolist()
            assert lens == [128, 128]
            # the routed decode over what is left, from summaries made anew, against the dense step where nothing is pruned
            q1 = torch.randn(b, h_q, d, generator=g).to(BF).to(DEV)
            o1, o2 = torch.empty_like(q1), torch.empty_like(q1)
            dp = B.params_for_paged_decode(q1, Kp, Vp, o1, max_pages=width, block=64, alpha=1.5, gamma=1e-6, sigma=1e8)
            kbar = B.alloc_kbar(dp)
            B.dash_attn_block_summaries_paged(dp, Kp, table, kbar, kv_len=new_len)
            dws = B.alloc_workspace(dp)
            B.dash_attn_fwd_decode_paged(dp, q1, Kp, Vp, table, kbar, new_len, o1, dws)
            p1 = B.params_for_paged(Kp, Vp, table, h_q=h_q, Q=q1, O=o2)
            B.dash_attn_attend_chunk_paged(p1, q1, Kp, Vp, table, dev([0, 1, 2]), new_len, o2, None, ws)
            assert (o1.float() - o2.float()).abs().max().item() < 2e-2


@pytest.mark.parametrize("dtype", [BF, F32])
def test_captured_graphs_replay_with_new_lengths(dtype):
    """The calls read lengths on the device: a captured step serves later lengths, and two graphs may share a workspace in turn."""
    c = Cache([1, 1], [300, 290], h_q=8, h_kv=2, d=128, page=64, dtype=dtype, width=5)
    mass = torch.zeros(2, 2, c.cap, device=DEV)
    c.attend()

    def step():
        B.dash_attn_attend_chunk_paged(c.p, c.Q, c.Kpool, c.Vpool, c.table, c.q_start, c.kv_len, c.O, c.lse, c.ws)
        B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, None, mass, c.ws)

    graphs = []
    for _ in range(2):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for k, lens in enumerate(([300, 290], [1, 257], [130, 64])):
        c.kv_lens = lens
        c.kv_len.copy_(torch.tensor(lens))
        for b in range(2):
            full = torch.arange(lens[b], device=DEV)
            c.Kc[b], c.Vc[b] = (t[c.table[b, full // 64].long(), full % 64].cpu() for t in (c.Kpool, c.Vpool))
        c.O.fill_(7.0)
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        assert B.dash_attn_last_status(c.ws) == 0
        c.check_attention()
        for b in range(2):
            assert abs(mass[b, :, :lens[b]].sum().item() - 8) < 1e-3


def test_two_streams_with_workspaces_of_their_own():
    cs = [Cache([1, 40], [3000 + 50 * k, 700], h_q=8, h_kv=2, d=128, page=64, dtype=BF, seed=k) for k in range(2)]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(cs, streams):
            with torch.cuda.stream(s):
                B.dash_attn_attend_chunk_paged(c.p, c.Q, c.Kpool, c.Vpool, c.table, c.q_start, c.kv_len, c.O, c.lse, c.ws)
    torch.cuda.synchronize()
    for c in cs:
        assert B.dash_attn_last_status(c.ws) == 0
        c.check_attention()


def test_calls_without_rows():
    """No new rows: append and attention do nothing, weights only decay."""
    for dtype in (BF, F32):
        c = Cache([0, 0], [100, 30], h_q=4, h_kv=2, d=64, page=32, dtype=dtype)
        assert c.rows == 0
        c.attend()
        e = torch.empty(0, 2, 64, dtype=dtype, device=DEV)
        B.dash_attn_append_paged(c.p, None, None, c.q_start, c.kv_len, c.table, None, None, e, e, c.Kpool, c.Vpool)
        mass = torch.rand(2, 2, c.cap, device=DEV)
        out = torch.full_like(mass, 9.0)
        B.dash_attn_key_mass_paged(c.p, c.Q, c.Kpool, c.table, c.q_start, c.kv_len, c.lse, mass, out, c.ws, decay=0.25)
        c.check_mass(mass, 0.25, out)


def test_types_and_devices_are_checked_before_the_launch():
    c = Cache([1], [10], h_q=2, h_kv=2, d=64, page=16, dtype=F32)
    with pytest.raises(ValueError):
        B.dash_attn_attend_chunk_paged(c.p, c.Q, c.Kpool, c.Vpool, c.table.long(), c.q_start, c.kv_len, c.O, c.lse, c.ws)
    with pytest.raises(ValueError):
        B.dash_attn_attend_chunk_paged(c.p, c.Q, c.Kpool, c.Vpool, c.table, c.q_start, c.kv_len, c.O, c.lse.double(), c.ws)
    with pytest.raises(ValueError):
        B.dash_attn_attend_chunk_paged(c.p, c.Q, c.Kpool.cpu(), c.Vpool, c.table, c.q_start, c.kv_len, c.O, c.lse, c.ws)
