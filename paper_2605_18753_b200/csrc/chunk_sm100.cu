// Dense causal attention of chunks of new tokens over a paged cache: tensor-core path for sm_100a (bf16).
//
//   o_i = sum_{t <= slot(i)} exp(s_it - m_i) v_t / l_i,   s_it = <q_i, k_t> / sqrt(d),
// one pass over the keys with a running maximum m and sum l per row.
//
// Unit of work: one (sequence, KV head) and up to 2 * TQ consecutive new tokens, TQ = 128 / g_q; the rows of an MMA tile are (token,
// head of the group) pairs, token-major, so all heads of a group share a K / V tile of 128 slots.  Two stages run against each
// other, each with a warpgroup for its softmax and a quarter-and-a-quarter of tensor memory (S 128 columns, O head_dim columns), so
// that one stage's MMAs hide the other's exponentials:
//   a unit of more than TQ tokens: stage 0 and 1 hold its two row tiles, and walk the same K / V tiles;
//   a unit of at most TQ tokens (decode): both stages hold the same rows and take every other K / V tile; their results are merged.
//
// Schedule: the K / V tiles of all units, one behind another, are cut into equal ranges, one per block (a persistent grid of one
// block per SM).  Sequences of any mix of lengths, one long cache or many short ones, keep every SM busy to the end.  A unit
// that is cut is finished by the last of its blocks to arrive, which merges the partial results (m, l, O) in the order of the cuts: the
// result does not depend on which block came last.  Only the two ends of a range can be cut, so partial results take two
// slots per block, whatever the problem.
//
// Warp roles (384 threads): warps 0-3 and 4-7 softmax of stage 0 / 1, a row per thread; warp 8 loads Q and K, warp 9 V (TMA, a box
// per page or per 128 tokens of one), warp 10 issues the MMAs, warp 11 completes the warpgroup for setmaxnreg.  P is written over S in
// tensor memory (bf16) and is the A operand of P V.
// Every wait is bounded; one that runs out raises DASH_ERR_TIMEOUT in the status word, and every role leaves.
#include <cuda.h>

#include "paged.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"

namespace dash {

namespace {

constexpr int NT = 128;                      // slots per K / V tile
constexpr int KST = 2, VST = 2;              // ring depths
constexpr int THREADS = 384;
constexpr int REGS_SOFTMAX = 208, REGS_SERVICE = 88;
static_assert(256 * REGS_SOFTMAX + 128 * REGS_SERVICE <= THREADS * 168, "what the block was launched with");
constexpr uint32_t TMEM_COLS = 512;          // S0 [0,128), S1 [128,256), O0 [256,256+d), O1 behind it
constexpr float RESCALE_LOG2 = 8.f;          // the running maximum moves only when it grew by more than this
constexpr int MAX_SLOTS = 4096;              // unit slots (see the plan) of one launch
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

enum Bar { Q_FULL = 0, Q_EMPTY, K_FULL, K_EMPTY = K_FULL + KST, V_FULL = K_EMPTY + KST, V_EMPTY = V_FULL + VST, S_FULL = V_EMPTY + VST,
           P_FULL = S_FULL + 2, PV_DONE = P_FULL + 2, O_FREE = PV_DONE + 2, MERGE = O_FREE + 2, N_BARS };

struct Misc {
  unsigned long long bar[N_BARS];
  uint32_t tmem_base;
  int abort_flag;
  int last;                                  // this block merges the unit
  int scan[THREADS / 32];
};

template <int HD>
struct Layout {
  static constexpr uint32_t Q_TILE = 128 * HD * 2;     // one row tile; regions of 64 elements (128 bytes, the swizzle span)
  static constexpr uint32_t KV_TILE = NT * HD * 2;
  static constexpr uint32_t OFF_K = 2 * Q_TILE;
  static constexpr uint32_t OFF_V = OFF_K + KST * KV_TILE;
  static constexpr uint32_t OFF_MISC = OFF_V + VST * KV_TILE;
  static constexpr uint32_t OFF_PLAN = (OFF_MISC + sizeof(Misc) + 15) / 16 * 16;
  static constexpr uint32_t smem(int slots) { return OFF_PLAN + (slots + 1) * 4 + slots * 2; }
  static_assert(OFF_PLAN + (MAX_SLOTS + 1) * 4 + MAX_SLOTS * 2 <= 232448, "one block per SM");
};

struct ChunkArgs {
  PagedDims pd;
  int TQ, slot0, n_slots;          // tokens per row tile; the launch's window of unit slots
  int box;                         // tokens per TMA box: divides the page and the tile
  int n_blocks;
  const int *q_start, *kv_len, *page_table;
  __nv_bfloat16* O;
  float* lse;
  float* partials;
  StatusBlock* sb;
};

// One block's share of a unit.
struct Piece {
  int b, r, t;                     // sequence, KV head, unit of the sequence
  int k0, len, n;                  // first K / V tile and number of them; the unit's
  long long f0;                    // the unit's first position in the list of all tiles
  Seq s;
  int tokens;                      // of the unit
  bool two;                        // two row tiles; else one, its K / V tiles in turns
};

// Slot of a sequence's unit: floor(q0 / TT) + b + t.  Each sequence has at least as many slots to itself as it has units
// (floor(x + y) + 1 - floor(x) >= ceil(y)), so the slot is known from q_start[b] alone; slots without a unit have no tiles.
struct Plan {
  const int* pref;                 // exclusive sums of the slots' tiles, and their total
  const unsigned short* seq;
  int total;                       // tiles per KV head
  long long all;
  long long begin, end;            // this block's range
};

__device__ __forceinline__ int unit_tiles(const PagedDims& pd, const Seq& s, int t, int TT) {
  const long long last = (long long)s.kv - s.q_len + min(s.q_len, (t + 1) * TT);      // slots up to the unit's last token's
  const int seen = (int)min(max(last, 0LL), (long long)s.valid);
  return max(1, (seen + NT - 1) / NT);       // a unit without a key still writes its rows
}

__device__ __forceinline__ Piece piece_at(const ChunkArgs& a, const Plan& pl, long long f) {
  Piece p;
  p.r = (int)(f / pl.total);
  const int rest = (int)(f - (long long)p.r * pl.total);
  int lo = 0, hi = a.n_slots;                // last slot with pref <= rest that has tiles
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pl.pref[mid] <= rest) lo = mid; else hi = mid;
  }
  p.b = pl.seq[lo];
  p.s = load_seq(a.pd, a.q_start, a.kv_len, p.b);
  const int TT = 2 * a.TQ;
  p.t = lo + a.slot0 - (p.s.q0 / TT + p.b);
  p.n = pl.pref[lo + 1] - pl.pref[lo];
  p.k0 = rest - pl.pref[lo];
  p.f0 = f - p.k0;
  p.len = (int)min((long long)(p.n - p.k0), pl.end - f);
  p.tokens = min(TT, p.s.q_len - p.t * TT);
  p.two = p.tokens > a.TQ;
  return p;
}

// Partial results of a block: slot 0 a unit begun by an earlier block, 1 one that a later block goes on with, 2 a whole unit in turns.
template <int HD> __host__ __device__ constexpr long long partial_floats() { return 128LL * (HD + 2); }
template <int HD>
__device__ __forceinline__ float* partial_at(const ChunkArgs& a, int block, int slot, int stage) {
  return a.partials + (((long long)block * 3 + slot) * 2 + stage) * partial_floats<HD>();
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

template <int HD>
__global__ void __launch_bounds__(THREADS, 1)
attend_chunk_sm100_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                          const __grid_constant__ CUtensorMap tmV, const __grid_constant__ ChunkArgs a) {
  using LY = Layout<HD>;
  extern __shared__ __align__(1024) uint8_t smem[];
  Misc* misc = reinterpret_cast<Misc*>(smem + LY::OFF_MISC);
  int* pref = reinterpret_cast<int*>(smem + LY::OFF_PLAN);
  unsigned short* slot_seq = reinterpret_cast<unsigned short*>(pref + a.n_slots + 1);
  const PagedDims& pd = a.pd;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sbase = ptx::smem_u32(smem);
  auto bar = [&](int i) { return ptx::smem_u32(&misc->bar[i]); };
  volatile int* abort_flag = &misc->abort_flag;
  auto wait_all = [&](uint32_t barrier, uint32_t parity) { return ptx::mbar_wait_warp(barrier, parity, abort_flag); };
  const int g_q = pd.g_q, TQ = a.TQ, TT = 2 * TQ;

  if (tid == 0) {
    misc->abort_flag = (sbase & 1023u) != 0u;
    for (int i = 0; i < N_BARS; ++i) ptx::mbar_init(bar(i), i >= P_FULL && i < PV_DONE ? 128 : i >= O_FREE && i < MERGE ? 128 : i == MERGE ? 256 : 1);
    ptx::fence_barrier_init();
  }
  if (warp == 10) {
    ptx::tmem_alloc(ptx::smem_u32(&misc->tmem_base), TMEM_COLS);
    ptx::tmem_relinquish();
    ptx::tc_fence_before();
  }
  for (int s = tid; s <= a.n_slots; s += THREADS) pref[s] = 0;
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = misc->tmem_base;
  chain_wait();
  if (a.sb && tid == 0) {
    const int old = *reinterpret_cast<volatile int*>(&a.sb->status);
    if (old != 0 || misc->abort_flag) {      // an earlier error on this workspace: leave at the first wait
      if (old == 0) report_error(a.sb, DASH_ERR_CUDA, 300);
      misc->abort_flag = 1;
    }
  }
  // ---- the plan: tiles of every unit of the window, then their sums
  for (int b = warp; b < pd.batch; b += THREADS / 32) {
    const Seq s = load_seq(pd, a.q_start, a.kv_len, b);
    const int base = s.q0 / TT + b - a.slot0, units = (s.q_len + TT - 1) / TT;
    for (int t = max(0, -base) + lane; t < units && base + t < a.n_slots; t += 32) {
      pref[base + t] = unit_tiles(pd, s, t, TT);
      slot_seq[base + t] = (unsigned short)b;
    }
  }
  __syncthreads();
  {
    const int per = (a.n_slots + THREADS - 1) / THREADS, s0 = min(tid * per, a.n_slots), s1 = min(s0 + per, a.n_slots);
    int sum = 0;
    for (int s = s0; s < s1; ++s) sum += pref[s];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) misc->scan[warp] = incl;
    __syncthreads();
    int run = incl - sum;
    for (int w = 0; w < warp; ++w) run += misc->scan[w];
    for (int s = s0; s < s1; ++s) {
      const int n = pref[s];
      pref[s] = run;
      run += n;
    }
    if (s1 == a.n_slots && s0 < s1) pref[a.n_slots] = run;
  }
  __syncthreads();
  Plan pl;
  pl.pref = pref;
  pl.seq = slot_seq;
  pl.total = pref[a.n_slots];
  pl.all = (long long)pl.total * pd.h_kv;
  // ranges of at least two tiles: fewer blocks where there is little to do
  const long long G = min((long long)a.n_blocks, max(1LL, (pl.all + 1) / 2));
  const int blk = blockIdx.x;
  pl.begin = blk < G ? blk * pl.all / G : 0;
  pl.end = blk < G ? (blk + 1) * pl.all / G : 0;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_SERVICE));
    if (warp == 8 || warp == 9) {
      // =========================== producers: K (and Q), V ===========================
      const bool is_k = warp == 8;
      const CUtensorMap* tm = is_k ? &tmK : &tmV;
      const uint32_t ring = sbase + (is_k ? LY::OFF_K : LY::OFF_V);
      const int full = is_k ? K_FULL : V_FULL, empty = is_k ? K_EMPTY : V_EMPTY;
      constexpr int ST = KST;
      static_assert(KST == VST, "one loop for both");
      const int boxes = NT / a.box;
      if (lane == 0) ptx::prefetch_tensormap(tm);
      int cnt = 0, q_cnt = 0;                 // tiles loaded; units
      bool ok = true;
      for (long long f = pl.begin; f < pl.end && ok;) {
        const Piece p = piece_at(a, pl, f);
        if (is_k) {
          if (q_cnt > 0) ok = wait_all(bar(Q_EMPTY), (q_cnt - 1) & 1);
          if (!ok) break;
          if (lane == 0) {
            const int tiles = p.two ? 2 : 1, row = p.s.q0 + p.t * TT;
            ptx::mbar_arrive_expect_tx(bar(Q_FULL), tiles * (HD / 64) * 128 * g_q * TQ);
            for (int s = 0; s < tiles; ++s)
              for (int h = 0; h < HD / 64; ++h)
                ptx::tma_load_4d(sbase + s * LY::Q_TILE + h * (LY::Q_TILE / (HD / 64)), &tmQ, bar(Q_FULL), h * 64, p.r * g_q, row + s * TQ, 0);
          }
          ++q_cnt;
        }
        const int* table = a.page_table + (long long)p.b * pd.max_pages;
        for (int j = 0; j < p.len && ok; ++j, ++cnt) {
          const int slot = (p.k0 + j) * NT + lane * a.box;
          int page = pd.num_pages, tok = 0;   // (out of range: the box is filled with zeros)
          if (lane < boxes && slot < p.s.valid) {
            const int lp = slot / pd.page_size;
            tok = slot - lp * pd.page_size;
            const int ph = __ldg(table + lp);
            if (ph >= 0 && ph < pd.num_pages) page = ph;
          }
          const int st = cnt % ST;
          if (cnt >= ST) ok = wait_all(bar(empty + st), (cnt / ST - 1) & 1);
          if (!ok) break;
          if (lane == 0) ptx::mbar_arrive_expect_tx(bar(full + st), LY::KV_TILE);
          __syncwarp();
          if (lane < boxes) {
            const uint32_t dst = ring + st * LY::KV_TILE + lane * a.box * 128;
#pragma unroll
            for (int h = 0; h < HD / 64; ++h)
              ptx::tma_load_4d(dst + h * (LY::KV_TILE / (HD / 64)), tm, bar(full + st), h * 64, p.r, tok, page);
          }
        }
        f += p.len;
      }
      // a wait ran out: let the copies already issued land (bounded) before the block retires
      if (!ok && lane == 0) {
        for (int c = max(0, cnt - ST); c < cnt; ++c)
          for (int k = 0; k < 200000 && !ptx::mbar_try_wait(bar(full + c % ST), (c / ST) & 1); ++k) {}
        if (is_k && q_cnt > 0)
          for (int k = 0; k < 200000 && !ptx::mbar_try_wait(bar(Q_FULL), (q_cnt - 1) & 1); ++k) {}
      }
    } else if (warp == 10) {
      // =========================== MMA issuer ===========================
      constexpr uint32_t IDESC_QK = ptx::idesc_bf16_f32(128, NT, false, false);
      constexpr uint32_t IDESC_PV = ptx::idesc_bf16_f32(128, HD, false, true);
      const uint64_t qd0 = ptx::smem_desc_sw128(sbase, 16, 1024);
      const uint64_t kd0 = ptx::smem_desc_sw128(sbase + LY::OFF_K, 16, 1024);
      const uint64_t vd0 = ptx::smem_desc_sw128(sbase + LY::OFF_V, NT * 128, 1024);
      const bool lead = ptx::elect_one();
      int base = 0, q_cnt = 0;                // K / V tiles of earlier pieces; pieces
      int it[2] = {0, 0};                     // steps of each stage so far
      bool ok = true;
      for (long long f = pl.begin; f < pl.end && ok;) {
        const Piece p = piece_at(a, pl, f);
        const int steps[2] = {p.two ? p.len : (p.len + 1) / 2, p.two ? p.len : p.len / 2};
        ok = wait_all(bar(Q_FULL), q_cnt & 1);
        if (!ok) break;
        auto tile_of = [&](int s, int i) { return base + (p.two ? i : 2 * i + s); };
        auto qk = [&](int s, int i) -> bool {
          const int c = tile_of(s, i), st = c % KST;
          if (!wait_all(bar(K_FULL + st), (c / KST) & 1)) return false;
          ptx::tc_fence_after();
          if (lead) {
            const uint64_t qd = qd0 + (uint64_t)((p.two && s ? LY::Q_TILE : 0u) >> 4);
            const uint64_t kd = kd0 + (uint64_t)((st * LY::KV_TILE) >> 4);
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {
              const uint64_t off = (uint64_t)(((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4);
              ptx::mma_bf16_ss(tmem + s * 128, qd + off, kd + off, IDESC_QK, k > 0 ? 1u : 0u);
            }
            ptx::mma_commit(bar(S_FULL + s));
            if (!p.two || s == 1) {
              ptx::mma_commit(bar(K_EMPTY + st));
              if (c == base + p.len - 1) ptx::mma_commit(bar(Q_EMPTY));      // the piece's last product with its queries
            }
          }
          __syncwarp();
          return true;
        };
        auto pv = [&](int s, int i) -> bool {
          const int c = tile_of(s, i), st = c % VST;
          if (!wait_all(bar(P_FULL + s), (it[s] + i) & 1)) return false;
          if (!wait_all(bar(V_FULL + st), (c / VST) & 1)) return false;
          // the first product of a unit overwrites O: its epilogue must have read the last one's
          if (i == 0 && q_cnt > 0 && !wait_all(bar(O_FREE + s), (q_cnt - 1) & 1)) return false;
          ptx::tc_fence_after();
          if (lead) {
            const uint64_t vd = vd0 + (uint64_t)((st * LY::KV_TILE) >> 4);
#pragma unroll
            for (int k = 0; k < NT / 16; ++k)
              ptx::mma_bf16_ts(tmem + 256 + s * HD, tmem + s * 128 + k * 8, vd + (uint64_t)((k * 16 * 128) >> 4), IDESC_PV, (i > 0 || k > 0) ? 1u : 0u);
            ptx::mma_commit(bar(PV_DONE + s));
            if (!p.two || s == 1) ptx::mma_commit(bar(V_EMPTY + st));
          }
          __syncwarp();
          return true;
        };
        ok = qk(0, 0) && (steps[1] == 0 || qk(1, 0));
        for (int i = 0; i < steps[0] && ok; ++i) {
          ok = pv(0, i) && (i + 1 >= steps[0] || qk(0, i + 1));
          if (ok && i < steps[1]) ok = pv(1, i) && (i + 1 >= steps[1] || qk(1, i + 1));
        }
        if (!ok) break;
        base += p.len;
        it[0] += steps[0];
        it[1] += steps[1];
        ++q_cnt;
        f += p.len;
      }
    }
  } else {
    // =========================== softmax, epilogue, merge ===========================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFTMAX));
    const int s = warp >> 2, m = tid & 127;            // stage; row of the tile = TMEM lane
    const int mt = m / g_q, hh = m - mt * g_q;         // token of the row tile, head of the group
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_addr = lane_addr + s * 128, o_addr = lane_addr + 256 + s * HD;
    const float c1 = pd.sm_scale * LOG2E;
    int base = 0, it = 0, merges = 0;
    bool ok = true;
    for (long long f = pl.begin; f < pl.end && ok;) {
      const Piece p = piece_at(a, pl, f);
      const int steps = p.two ? p.len : s == 0 ? (p.len + 1) / 2 : p.len / 2;
      const int first = p.two && s ? TQ : 0;           // first token of this stage's rows in the unit
      const int i_row = p.t * TT + first + mt;
      const bool row_on = mt < TQ && first + mt < p.tokens;
      const bool warp_on = __any_sync(0xffffffffu, row_on);
      // slots that the row sees (rows that are not there never ask for a mask)
      const int seen = !row_on ? 0x7fffffff : (int)min(max((long long)p.s.kv - p.s.q_len + i_row + 1, 0LL), (long long)p.s.valid);
      float m_used = -INFINITY, l = 0.f;
      for (int i = 0; i < steps; ++i) {
        const int j = p.two ? i : 2 * i + s, kv0 = (p.k0 + j) * NT, c = base + j;
        ok = wait_all(bar(S_FULL + s), (it + i) & 1);      // (the stage's product with V of the step before is done as well)
        if (!ok) break;
        // Stale rows behind the cache's end must not meet P = 0 as NaN: they are cleared in the tile.  (Not before the wait above: the
        // tile before in this place of the ring may not even have arrived, and the phase bit could not tell its load from this one's.)
        if (kv0 + NT > p.s.valid) {
          ok = wait_all(bar(V_FULL + c % VST), (c / VST) & 1);
          if (!ok) break;
          if (kv0 + m >= p.s.valid) {
            uint8_t* row = smem + LY::OFF_V + (c % VST) * LY::KV_TILE + m * 128;
#pragma unroll
            for (int h = 0; h < HD / 64; ++h)
#pragma unroll
              for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4*>(row + h * (NT * 128) + q * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          ptx::fence_proxy_async_smem();
        }
        if (warp_on) {
          ptx::tc_fence_after();
          uint32_t sr[128];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t* part = sr + 32 * q;
            DASH_TMEM_LD32(part, s_addr + 32 * q);
          }
          ptx::tmem_wait_ld();
          const int vis = seen - kv0;
          if (__any_sync(0xffffffffu, vis < NT)) {
#pragma unroll
            for (int k = 0; k < NT; ++k)
              if (k >= vis) sr[k] = 0xff800000u;       // -inf
          }
          float ch[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) ch[k] = __uint_as_float(sr[k]);
#pragma unroll
          for (int q = 8; q + 16 <= NT; q += 16)
#pragma unroll
            for (int k = 0; k < 8; ++k) ch[k] = max3(ch[k], __uint_as_float(sr[q + k]), __uint_as_float(sr[q + k + 8]));
#pragma unroll
          for (int k = 0; k < 8; ++k) ch[k] = fmaxf(ch[k], __uint_as_float(sr[NT - 8 + k]));
          const float top = fmaxf(max3(ch[0], ch[1], ch[2]), fmaxf(max3(ch[3], ch[4], ch[5]), fmaxf(ch[6], ch[7]))) * c1;
          float corr = 1.f;
          bool moved = false;
          if (top > m_used + RESCALE_LOG2 || (m_used == -INFINITY && top > -INFINITY)) {
            corr = exp2f(m_used - top);                // 0 when nothing was accumulated yet
            m_used = top;
            moved = true;
          }
          l *= corr;
          // (O is stable: the scores' barrier also stands for every product issued before them)
          if (__any_sync(0xffffffffu, moved) && i > 0) {
#pragma unroll 1
            for (int q = 0; q < HD / 32; ++q) {
              uint32_t o[32];
              DASH_TMEM_LD32(o, o_addr + q * 32);
              ptx::tmem_wait_ld();
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * corr);
              DASH_TMEM_ST32(o_addr + q * 32, o);
            }
          }
          const float off = m_used == -INFINITY ? 0.f : -m_used;
          const float2 c1v = make_float2(c1, c1), offv = make_float2(off, off);
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t pk[16];
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              const float2 x = __ffma2_rn(make_float2(__uint_as_float(sr[32 * q + k]), __uint_as_float(sr[32 * q + k + 1])), c1v, offv);
              const float2 e = make_float2(exp2f(x.x), exp2f(x.y));
              sum[(k >> 1) & 1] = __fadd2_rn(sum[(k >> 1) & 1], e);
              const __nv_bfloat162 hv = __floats2bfloat162_rn(e.x, e.y);
              pk[k >> 1] = *reinterpret_cast<const uint32_t*>(&hv);
            }
            ptx::tmem_st_n<16>(s_addr + 16 * q, pk);
          }
          const float2 ls = __fadd2_rn(sum[0], sum[1]);
          l += ls.x + ls.y;
          ptx::tmem_wait_st();
          ptx::tc_fence_before();
        }
        ptx::mbar_arrive(bar(P_FULL + s));
      }
      if (!ok) break;
      // ---- the unit's rows, or what this block has of them
      if (steps > 0) {
        ok = wait_all(bar(PV_DONE + s), (it + steps - 1) & 1);
        if (!ok) break;
        ptx::tc_fence_after();
      }
      const bool whole = p.len == p.n;
      const long long row = (long long)p.s.q0 + i_row, head = (long long)p.r * g_q + hh;
      auto lse_of = [&](float mx, float sm) { return sm > 0.f ? (mx + __log2f(sm)) * LN2 : -INFINITY; };
      auto pack4 = [](float x, float y, float z, float w) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(x, y), hi = __floats2bfloat162_rn(z, w);
        return make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      };
      if (whole && p.two) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
        __nv_bfloat16* op = a.O + row * pd.os[0] + head * pd.os[1];
#pragma unroll 1
        for (int q = 0; q < HD / 32 && warp_on; ++q) {
          __syncwarp();                                // (rows that are not there skipped the stores of the round before)
          uint32_t o[32];
          DASH_TMEM_LD32(o, o_addr + q * 32);
          ptx::tmem_wait_ld();
          if (row_on) {
#pragma unroll
            for (int k = 0; k < 32; k += 8) {
              float x[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(o[k + e]) * inv;
              const uint2 lo = pack4(x[0], x[1], x[2], x[3]), hi = pack4(x[4], x[5], x[6], x[7]);
              *reinterpret_cast<uint4*>(op + q * 32 + k) = make_uint4(lo.x, lo.y, hi.x, hi.y);
            }
          }
        }
        if (row_on && a.lse) a.lse[row * pd.h_q + head] = lse_of(m_used, l);
        ptx::tc_fence_before();
        ptx::mbar_arrive(bar(O_FREE + s));
      } else {
        // partial result: O unnormalised, four columns of all rows one behind another, then (m, l)
        const int slot = whole ? 2 : p.k0 > 0 ? 0 : 1;
        float* part = partial_at<HD>(a, blk, slot, s);
        if (warp_on) {
#pragma unroll 1
          for (int q = 0; q < HD / 32 && steps > 0; ++q) {
            __syncwarp();
            uint32_t o[32];
            DASH_TMEM_LD32(o, o_addr + q * 32);
            ptx::tmem_wait_ld();
            if (row_on) {
#pragma unroll
              for (int k = 0; k < 32; k += 4)
                __stcg(reinterpret_cast<float4*>(part) + (long long)((q * 32 + k) >> 2) * 128 + m,
                       make_float4(__uint_as_float(o[k]), __uint_as_float(o[k + 1]), __uint_as_float(o[k + 2]), __uint_as_float(o[k + 3])));
            }
          }
          if (row_on) __stcg(reinterpret_cast<float2*>(part + 128 * HD) + m, make_float2(m_used, l));
        }
        ptx::tc_fence_before();
        ptx::mbar_arrive(bar(O_FREE + s));
        __threadfence();
        auto meet = [&]() {
          ptx::mbar_arrive(bar(MERGE));
          return wait_all(bar(MERGE), merges++ & 1);
        };
        if (!(ok = meet())) break;
        // blocks of the unit, in order: those whose ranges hold its first and its last tile
        const int c1st = (int)(((p.f0 + 1) * G - 1) / pl.all), cend = (int)(((p.f0 + p.n) * G - 1) / pl.all);
        bool last = true;
        if (!whole) {
          if (tid == 0) {
            __threadfence();                           // the block's results, which meet() has gathered, before the count
            int* counter = arrival_counters(a.sb) + c1st;
            const bool is_last = atomicAdd(counter, 1) == cend - c1st;
            if (is_last) *counter = 0;
            __threadfence();
            misc->last = is_last;
          }
          if (!(ok = meet())) break;
          last = *reinterpret_cast<volatile int*>(&misc->last) != 0;
          __threadfence();
        }
        if (last) {
          // two row tiles: each warpgroup merges its own; else both share the rows, and every block has two parts of them
          const int tokens = p.two ? min(TQ, p.tokens - first) : p.tokens, rows = tokens * g_q;
          const int per = p.two ? 1 : 2, parts = (cend - c1st + 1) * per;
          auto part_of = [&](int k) {
            const int cb = c1st + k / per;
            return partial_at<HD>(a, cb, whole ? 2 : cb == c1st ? 1 : 0, p.two ? s : k % per);
          };
          for (int e = p.two ? m : tid; e < rows * (HD / 4); e += p.two ? 128 : 256) {
            const int mr = e % rows, c4 = e / rows;
            float mx = -INFINITY, sm = 0.f;
            for (int k = 0; k < parts; ++k) mx = fmaxf(mx, __ldcg(reinterpret_cast<const float2*>(part_of(k) + 128 * HD) + mr).x);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
            for (int k = 0; k < parts; ++k) {
              const float* src = part_of(k);
              const float2 ml = __ldcg(reinterpret_cast<const float2*>(src + 128 * HD) + mr);
              if (ml.x > -INFINITY) {
                const float w = exp2f(ml.x - mx);
                const float4 o = __ldcg(reinterpret_cast<const float4*>(src) + (long long)c4 * 128 + mr);
                sm = fmaf(ml.y, w, sm);
                acc.x = fmaf(o.x, w, acc.x); acc.y = fmaf(o.y, w, acc.y);
                acc.z = fmaf(o.z, w, acc.z); acc.w = fmaf(o.w, w, acc.w);
              }
            }
            const float inv = sm > 0.f ? 1.f / sm : 0.f;
            const int mtok = mr / g_q, mh = mr - mtok * g_q;
            const long long orow = (long long)p.s.q0 + p.t * TT + first + mtok, ohead = (long long)p.r * g_q + mh;
            *reinterpret_cast<uint2*>(a.O + orow * pd.os[0] + ohead * pd.os[1] + c4 * 4) = pack4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
            if (c4 == 0 && a.lse) a.lse[orow * pd.h_q + ohead] = lse_of(mx, sm);
          }
        }
        // slot 2 is written again by this block's next such unit
        if (whole && !(ok = meet())) break;
      }
      base += p.len;
      it += steps;
      f += p.len;
    }
    ptx::tc_fence_before();
  }

  __syncthreads();
  if (warp == 10) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, TMEM_COLS);
  }
  if (tid == 0 && misc->abort_flag) report_error(a.sb, DASH_ERR_TIMEOUT, 301);
}

// 4-D map of rows [outer][inner][heads][d]: the pool (pages, tokens, heads) or the packed queries (one page of rows).
bool make_map(CUtensorMap* out, const void* base, int d, int heads, long long tokens, long long pages, long long s_head, long long s_tok,
              long long s_page, int box_heads, int box_tokens) {
  cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)tokens, (cuuint64_t)pages};
  auto st = [](long long e) { return (cuuint64_t)((e > 0 ? e : 8) * 2); };      // a dimension of size 1 may have any stride
  cuuint64_t strides[3] = {st(s_head), st(s_tok), st(s_page)};
  cuuint32_t box[4] = {64u, (cuuint32_t)box_heads, (cuuint32_t)box_tokens, 1u};
  return encode_bf16_sw128_4d(out, base, dims, strides, box);
}

template <int HD>
cudaError_t launch_hd(ChunkArgs& a, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, cudaStream_t st) {
  auto kern = attend_chunk_sm100_kernel<HD>;
  static std::atomic<unsigned long long> configured{0};
  if (cudaError_t e = allow_dynamic_smem(kern, Layout<HD>::smem(MAX_SLOTS), configured); e != cudaSuccess) return e;
  const long long slots = a.pd.rows / (2 * a.TQ) + (long long)a.pd.batch;
  for (long long s0 = 0; s0 < slots; s0 += MAX_SLOTS) {
    a.slot0 = (int)s0;
    a.n_slots = (int)(slots - s0 < MAX_SLOTS ? slots - s0 : MAX_SLOTS);
    cudaError_t e = launch_chained(kern, dim3((unsigned)a.n_blocks), dim3(THREADS), Layout<HD>::smem(a.n_slots), st, tq, tk, tv, a);
    count_launch();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

bool paged_pool_map(void* map, const PagedDims& pd, const void* pool, const long long* s, int box) {
  return make_map(static_cast<CUtensorMap*>(map), pool, pd.d, pd.h_kv, pd.page_size, pd.num_pages, s[2], s[1], s[0], 1, box);
}
bool paged_q_map(void* map, const PagedDims& pd, const void* Q, int box_tokens) {
  return make_map(static_cast<CUtensorMap*>(map), Q, pd.d, pd.h_q, pd.rows, 1, pd.qs[1], pd.qs[0], 0, pd.g_q, box_tokens);
}
int paged_box(const PagedDims& pd) {
  int box = 128;
  while (pd.page_size % box) box >>= 1;
  return box;
}

bool chunk_sm100_supported(const PagedDims& pd) {
  // tensor maps have no stride of 0 over several elements
  auto rep = [](long long s, long long n) { return s == 0 && n > 1; };
  if (rep(pd.qs[0], pd.rows) || rep(pd.qs[1], pd.h_q)) return false;
  if (rep(pd.ks[0], pd.num_pages) || rep(pd.ks[1], pd.page_size) || rep(pd.ks[2], pd.h_kv)) return false;
  if (rep(pd.vs[0], pd.num_pages) || rep(pd.vs[1], pd.page_size) || rep(pd.vs[2], pd.h_kv)) return false;
  return tensor_map_encoder() != nullptr;
}

// Two row tiles in three slots of every block; as many blocks as the arrival counters could serve.
size_t chunk_sm100_partial_bytes(const PagedDims& pd) {
  return (size_t)256 * 6 * (size_t)(pd.d == 128 ? partial_floats<128>() : partial_floats<64>()) * sizeof(float);
}

cudaError_t launch_attend_chunk_sm100(const PagedDims& pd, const void* Q, const void* Kpool, const void* Vpool,
                                      const int* page_table, const int* q_start, const int* kv_len, void* O, float* lse,
                                      float* partials, StatusBlock* sb, cudaStream_t st) {
  ChunkArgs a;
  a.pd = pd;
  a.TQ = 128 / pd.g_q;
  a.box = paged_box(pd);
  a.n_blocks = current_sm_count() < 256 ? current_sm_count() : 256;
  a.q_start = q_start; a.kv_len = kv_len; a.page_table = page_table;
  a.O = (__nv_bfloat16*)O;
  a.lse = lse;
  a.partials = partials;
  a.sb = sb;
  CUtensorMap tq, tk, tv;
  if (!paged_q_map(&tq, pd, Q, a.TQ) || !paged_pool_map(&tk, pd, Kpool, pd.ks, a.box) || !paged_pool_map(&tv, pd, Vpool, pd.vs, a.box))
    return cudaErrorInvalidValue;
  return pd.d == 128 ? launch_hd<128>(a, tq, tk, tv, st) : launch_hd<64>(a, tq, tk, tv, st);
}

}  // namespace dash
