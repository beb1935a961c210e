// Attention weight per cached token, summed over a chunk's rows and a group's heads: tensor-core path for sm_100a (bf16).
//
//   mass_t = decay * mass_t + sum over rows (i, h) with slot(i) >= t of exp(s_iht - lse_ih),     s = <q, k_t> / sqrt(d).
// The rows' log-sum-exps are known, so a weight needs no running maximum: the scores are formed transposed, S^T = K Q^T, and a
// thread that owns a slot (a TMEM lane) adds up its row of exponentials.  No exchange between threads, no atomics, one order.
//
// Unit of work: one (sequence, KV head) and 256 slots, two K tiles of 128 that stay in shared memory while the query tiles (NQ
// (token, head) columns) go by; each has two S buffers in tensor memory, so the MMAs of a tile run while the exponentials of the one
// before are taken.  NQ = 128, or 16 for calls with few new tokens per sequence (decode), which stream K.
// A step of 128 columns is bound by its 32768 exponentials: 2048 clocks of the exponential unit (16 a clock), 1536 with every fourth pair
// on the FMA pipe as they are now; two warpgroups share a K tile's columns (four warps on a scheduler, so that one's waits are
// covered by the others'; with two, a step took 2600 clocks).
//
// Schedule: the (unit, query tile) steps of all units, one behind another, are cut into equal ranges, one per block of a persistent
// grid.  A cut unit's sums go to a place per block and end, and a second kernel adds them up in the order of the cuts.
//
// Warp roles: 16 warps of sums (8 where NQ = 16); then a warp that loads K (two units deep) and Q tiles, one for the log-sum-exps
// and slots of the columns, one that issues the MMAs, and one that completes the warpgroup.  Every wait is bounded
// (DASH_ERR_TIMEOUT in the status word).
#include <cuda.h>

#include "paged.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"

namespace dash {

bool paged_pool_map(void* map, const PagedDims& pd, const void* pool, const long long* s, int box);
bool paged_q_map(void* map, const PagedDims& pd, const void* Q, int box_tokens);
int paged_box(const PagedDims& pd);

namespace {

constexpr int NT = 128, PAIR = 256;          // slots per K tile, per unit
constexpr uint32_t TMEM_COLS = 512;          // [K tile][S buffer] of 128 columns
constexpr int MAX_SEQS = 2048;               // sequences of one launch
constexpr float LOG2E = 1.4426950408889634f;

enum Bar { Q_FULL = 0, Q_EMPTY = 2, L_FULL = 4, S_FULL = 6, S_EMPTY = 10, R_FULL = 14, R_EMPTY = 16, K_FULL = 18, K_EMPTY = 21, DRAIN = 24, N_BARS };

// Warpgroups of sums per K tile, and threads of a block.
template <int NQ> constexpr int GROUPS = NQ == 128 ? 2 : 1;
template <int NQ> constexpr int THREADS = 256 * GROUPS<NQ> + 128;

struct Misc {
  unsigned long long bar[N_BARS];
  uint32_t tmem_base;
  int abort_flag;
  __align__(16) float neg_lse[2][128];       // -lse * log2(e) of the columns (-inf: no weight)
  __align__(16) int slot[2][128];            // slots of the columns; -1: no row
  float half[2][128];                        // sums of a K tile's second warpgroup
  long long scan[20];
};

// K: KB units deep, [unit][tile]; regions of 64 elements (128 bytes) per row.  Where the query tiles are small a third unit fits.
template <int HD, int NQ>
struct Layout {
  static constexpr int KB = NQ == 128 ? 2 : 3;
  static constexpr uint32_t TILE = NT * HD * 2;
  static constexpr uint32_t Q_HALF = NQ * 128, Q_TILE = HD / 64 * Q_HALF;
  static constexpr uint32_t OFF_Q = KB * 2 * TILE;
  static constexpr uint32_t OFF_MISC = OFF_Q + 2 * Q_TILE;
  static constexpr uint32_t OFF_PLAN = (OFF_MISC + sizeof(Misc) + 15) / 16 * 16;
  static constexpr uint32_t smem(int seqs) { return OFF_PLAN + (seqs + 1) * 8; }
  static_assert(OFF_PLAN + (MAX_SEQS + 1) * 8 <= 232448, "one block per SM");
};

struct MassArgs {
  PagedDims pd;
  int QT, box, seq0, n_seqs;       // tokens per query tile; tokens per K box; the launch's sequences
  const int *q_start, *kv_len, *page_table;
  const float *lse, *mass_in;
  float* mass_out;
  float decay;
  float* parts;                    // [block][place][256]: place 0 a unit begun by an earlier block, 1 one that later blocks go on with
  struct MassCut* cuts;
  StatusBlock* sb;
  int inject;                      // test hook: the keys of a block's second unit are never loaded (the waits for them run out)
  long long wait_limit;            // clocks that a bounded wait may spin
};

struct MassCut {                   // the unit that a block cuts at its end
  int blocks, b, r, slot0;         // blocks that hold a part of it (0: none is cut)
};

// Which pairs of columns take their exponentials on the FMA pipe (exp2_fma): every fourth of a 128-column step (2048 rows over 8192
// slots, 32/8 heads, d 128: none 144 us, one in eight or in four 139.5, three in eight 143); none where K is streamed.
template <int STEP> __host__ __device__ constexpr bool on_fma(int pair) { return STEP == 32 && pair % 4 == 3; }

// A sequence's units: query tiles, KV heads apart; unit k begins at slot k * PAIR and is seen by the tiles from first_tile on.
struct SeqUnits {
  Seq s;
  int units, tiles, full;          // per KV head; units that all tiles see
  __device__ __forceinline__ SeqUnits() {}
  __device__ __forceinline__ SeqUnits(const MassArgs& a, int b) : s(load_seq(a.pd, a.q_start, a.kv_len, b)) {
    units = (s.valid + PAIR - 1) / PAIR;
    tiles = (s.q_len + a.QT - 1) / a.QT;
    const long long old = (long long)s.kv - s.q_len;
    full = old < 0 ? 0 : (int)min((long long)units, old / PAIR + 1);
  }
  __device__ __forceinline__ int first_tile(const MassArgs& a, int k) const {
    if (k < full) return 0;
    const long long i0 = (long long)k * PAIR - ((long long)s.kv - s.q_len);      // first token that sees the unit's first slot
    return i0 >= s.q_len ? tiles : (int)i0 / a.QT;
  }
  __device__ __forceinline__ int steps(const MassArgs& a, int k) const { return max(1, tiles - first_tile(a, k)); }      // (1: nothing to add, but to write)
  __device__ __forceinline__ long long head_steps(const MassArgs& a) const {
    long long n = (long long)full * max(1, tiles);
    for (int k = full; k < units; ++k) n += steps(a, k);
    return n;
  }
};

// The pieces of a block's range, in order.
struct MassWalk {
  long long left;                  // steps left of the range
  int b, r, k, t, n;               // sequence (of the launch's), KV head, unit, first step of the piece in the unit, the unit's steps
  SeqUnits u;
  __device__ __forceinline__ MassWalk(const MassArgs& a, const long long* pref, long long begin, long long end) {
    left = end - begin;
    b = r = k = t = n = 0;
    if (left <= 0) return;
    int lo = 0, hi = a.n_seqs;                 // last sequence with pref <= begin that has steps
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pref[mid] <= begin) lo = mid; else hi = mid;
    }
    b = lo;
    u = SeqUnits(a, a.seq0 + b);
    const long long per = (pref[b + 1] - pref[b]) / a.pd.h_kv;
    long long rest = begin - pref[b];
    r = (int)(rest / per);
    rest -= r * per;
    const int tiles = max(1, u.tiles);
    k = (int)min(rest / tiles, (long long)u.full);
    rest -= (long long)k * tiles;
    if (k == u.full)
      for (; rest >= u.steps(a, k); ++k) rest -= u.steps(a, k);
    t = (int)rest;
    n = u.steps(a, k);
  }
  __device__ __forceinline__ int len() const { return (int)min((long long)(n - t), left); }
  __device__ __forceinline__ bool done() const { return left <= 0; }
  __device__ __forceinline__ void next(const MassArgs& a, const long long* pref) {
    left -= len();
    t = 0;
    if (left <= 0) return;
    if (++k == u.units) {
      k = 0;
      if (++r == a.pd.h_kv) {
        r = 0;
        do ++b; while (pref[b + 1] == pref[b]);
        u = SeqUnits(a, a.seq0 + b);
      }
    }
    n = u.steps(a, k);
  }
};

struct Unit {
  int b, r, slot0;                 // first slot
  int t0, t1;                      // query tiles of the piece (none: t0 == t1)
  bool whole;
  const Seq& s;
  __device__ __forceinline__ Unit(const MassArgs& a, const MassWalk& w) : s(w.u.s) {
    b = a.seq0 + w.b;
    r = w.r;
    slot0 = w.k * PAIR;
    t0 = w.u.first_tile(a, w.k) + w.t;
    t1 = min(t0 + w.len(), w.u.tiles);
    whole = w.len() == w.n;
  }
};

// Adds the weights of one slot (a TMEM lane) in STEP columns, scores `sr`.  MASKED: some column is no row, or a row that does not see
// the slot.  (Two copies: a condition inside would cost its instructions in every column.)
template <int STEP, bool MASKED>
__device__ __forceinline__ void add_columns(float2 (&sum)[4], const uint32_t* sr, float2 scale, const float* neg_lse, const int* slots, int slot) {
#pragma unroll
  for (int c = 0; c < STEP; c += 4) {
    const float4 nl = *reinterpret_cast<const float4*>(neg_lse + c);
    const float2 e0 = __ffma2_rn(make_float2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])), scale, make_float2(nl.x, nl.y));
    const float2 e1 = __ffma2_rn(make_float2(__uint_as_float(sr[c + 2]), __uint_as_float(sr[c + 3])), scale, make_float2(nl.z, nl.w));
    float2 w0 = on_fma<STEP>(c >> 1) ? exp2_fma(e0) : make_float2(exp2f(e0.x), exp2f(e0.y));
    float2 w1 = on_fma<STEP>((c >> 1) + 1) ? exp2_fma(e1) : make_float2(exp2f(e1.x), exp2f(e1.y));
    if (MASKED) {
      const int4 sl = *reinterpret_cast<const int4*>(slots + c);
      if (sl.x < slot) w0.x = 0.f;
      if (sl.y < slot) w0.y = 0.f;
      if (sl.z < slot) w1.x = 0.f;
      if (sl.w < slot) w1.y = 0.f;
    }
    sum[(c >> 1) & 2] = __fadd2_rn(sum[(c >> 1) & 2], w0);
    sum[((c >> 1) & 2) + 1] = __fadd2_rn(sum[((c >> 1) & 2) + 1], w1);
  }
}

__device__ __forceinline__ long long mass_at(const MassArgs& a, int b, int r, int slot) { return ((long long)b * a.pd.h_kv + r) * a.pd.cap + slot; }
__device__ __forceinline__ float old_mass(const MassArgs& a, int b, int r, int slot, const Seq& s) {
  return a.mass_in && (long long)slot < (long long)s.kv - s.q_len ? a.decay * a.mass_in[mass_at(a, b, r, slot)] : 0.f;
}

template <int HD, int NQ>
__global__ void __launch_bounds__(THREADS<NQ>, 1)
key_mass_sm100_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ MassArgs a) {
  using LY = Layout<HD, NQ>;
  constexpr int STEP = NQ < 32 ? NQ : 32;    // columns of one tensor-memory load
  extern __shared__ __align__(1024) uint8_t smem[];
  Misc* misc = reinterpret_cast<Misc*>(smem + LY::OFF_MISC);
  long long* pref = reinterpret_cast<long long*>(smem + LY::OFF_PLAN);
  const PagedDims& pd = a.pd;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sbase = ptx::smem_u32(smem);
  auto bar = [&](int i) { return ptx::smem_u32(&misc->bar[i]); };
  volatile int* abort_flag = &misc->abort_flag;
  auto wait_all = [&](uint32_t barrier, uint32_t parity) { return ptx::mbar_wait_warp(barrier, parity, abort_flag, a.wait_limit); };
  const int g_q = pd.g_q, QT = a.QT;

  if (tid == 0) {
    misc->abort_flag = (sbase & 1023u) != 0u;
    for (int i = 0; i < N_BARS; ++i)
      ptx::mbar_init(bar(i), i >= K_FULL ? 1 : i >= R_FULL ? 4 : i >= S_EMPTY ? 4 * GROUPS<NQ> : 1);      // one arrival per warp
    ptx::fence_barrier_init();
  }
  constexpr int SUM_WARPS = 8 * GROUPS<NQ>;
  if (warp == SUM_WARPS + 2) {
    ptx::tmem_alloc(ptx::smem_u32(&misc->tmem_base), TMEM_COLS);
    ptx::tmem_relinquish();
    ptx::tc_fence_before();
  }
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = misc->tmem_base;
  chain_wait();
  if (a.sb && tid == 0) {
    const int old = *reinterpret_cast<volatile int*>(&a.sb->status);
    if (old != 0 || misc->abort_flag) {      // an earlier error on this workspace: leave at the first wait
      if (old == 0) report_error(a.sb, DASH_ERR_CUDA, 310);
      misc->abort_flag = 1;
    }
  }
  // ---- the plan: steps of every sequence, summed
  {
    const int per = (a.n_seqs + THREADS<NQ> - 1) / THREADS<NQ>, s0 = min(tid * per, a.n_seqs), s1 = min(s0 + per, a.n_seqs);
    long long sum = 0;
    for (int s = s0; s < s1; ++s) {
      const long long steps = SeqUnits(a, a.seq0 + s).head_steps(a) * pd.h_kv;
      pref[s] = steps;
      sum += steps;
    }
    long long incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) misc->scan[warp] = incl;
    __syncthreads();
    long long run = incl - sum;
    for (int w = 0; w < warp; ++w) run += misc->scan[w];
    for (int s = s0; s < s1; ++s) {
      const long long n = pref[s];
      pref[s] = run;
      run += n;
    }
    if (s1 == a.n_seqs && s0 < s1) pref[a.n_seqs] = run;
  }
  __syncthreads();
  const long long all = pref[a.n_seqs], G = min((long long)gridDim.x, max(1LL, all));
  const int blk = blockIdx.x;
  const long long begin = blk < G ? blk * all / G : 0;
  MassWalk walk(a, pref, begin, blk < G ? (blk + 1) * all / G : 0);

  if (warp == SUM_WARPS) {
    // =========================== K and Q tiles ===========================
    const int boxes = PAIR / a.box, per_tile = NT / a.box;
    if (lane == 0) {
      ptx::prefetch_tensormap(&tmQ);
      ptx::prefetch_tensormap(&tmK);
    }
    int kc = 0, qc = 0;
    bool ok = true;
    for (; ok && !walk.done(); walk.next(a, pref)) {
      const Unit x(a, walk);
      if (x.t0 >= x.t1) continue;
      if (a.inject && kc == 1) break;
      const int* table = a.page_table + (long long)x.b * pd.max_pages;
      const int slot = x.slot0 + lane * a.box;
      int page = pd.num_pages, tok = 0;      // (out of range: zeros)
      if (lane < boxes && slot < x.s.valid) {
        const int lp = slot / pd.page_size;
        tok = slot - lp * pd.page_size;
        const int ph = __ldg(table + lp);
        if (ph >= 0 && ph < pd.num_pages) page = ph;
      }
      const int kb = kc % LY::KB;
      if (kc >= LY::KB) ok = wait_all(bar(K_EMPTY + kb), (kc / LY::KB - 1) & 1);
      if (!ok) break;
      if (lane == 0) ptx::mbar_arrive_expect_tx(bar(K_FULL + kb), 2 * LY::TILE);
      __syncwarp();
      if (lane < boxes) {
        const uint32_t dst = sbase + (kb * 2 + lane / per_tile) * LY::TILE + (lane % per_tile) * a.box * 128;
#pragma unroll
        for (int h = 0; h < HD / 64; ++h) ptx::tma_load_4d(dst + h * (NT * 128), &tmK, bar(K_FULL + kb), h * 64, x.r, tok, page);
      }
      ++kc;
      for (int t = x.t0; t < x.t1 && ok; ++t, ++qc) {
        const int qb = qc & 1;
        if (qc >= 2) ok = wait_all(bar(Q_EMPTY + qb), (qc / 2 - 1) & 1);
        if (!ok) break;
        if (lane == 0) {
          ptx::mbar_arrive_expect_tx(bar(Q_FULL + qb), (HD / 64) * 128 * g_q * QT);
          for (int h = 0; h < HD / 64; ++h)
            ptx::tma_load_4d(sbase + LY::OFF_Q + qb * LY::Q_TILE + h * LY::Q_HALF, &tmQ, bar(Q_FULL + qb), h * 64, x.r * g_q, x.s.q0 + t * QT, 0);
        }
      }
    }
    if (lane == 0) {               // where a wait has run out, here or in another warp, the copies already issued land (bounded) first
      for (int c = max(0, kc - LY::KB); c < kc; ++c)
        for (int k = 0; k < 200000 && !ptx::mbar_try_wait(bar(K_FULL + c % LY::KB), (c / LY::KB) & 1); ++k) {}
      for (int c = max(0, qc - 2); c < qc; ++c)
        for (int k = 0; k < 200000 && !ptx::mbar_try_wait(bar(Q_FULL + (c & 1)), (c / 2) & 1); ++k) {}
    }
  } else if (warp == SUM_WARPS + 1) {
    // =========================== log-sum-exps and slots of the columns ===========================
    int qc = 0;
    bool ok = true;
    for (; ok && !walk.done(); walk.next(a, pref)) {
      const Unit x(a, walk);
      for (int t = x.t0; t < x.t1 && ok; ++t, ++qc) {
        const int qb = qc & 1;
        float v[NQ / 16];
        int at[NQ / 16];
#pragma unroll
        for (int k = 0; k < (NQ + 31) / 32; ++k) {
          const int c = lane + 32 * k, mt = c / g_q, hh = c - mt * g_q, i = t * QT + mt;
          v[k] = -INFINITY;
          at[k] = -1;
          if (c < NQ && mt < QT && i < x.s.q_len) {
            const float e = __ldg(a.lse + (long long)(x.s.q0 + i) * pd.h_q + x.r * g_q + hh);
            if (e > -INFINITY) v[k] = -e * LOG2E;
            at[k] = (int)min((long long)x.s.kv - x.s.q_len + i, (long long)0x7fffffff);
          }
        }
        if (qc >= 2) ok = wait_all(bar(S_EMPTY + qb), (qc / 2 - 1) & 1) && wait_all(bar(S_EMPTY + 2 + qb), (qc / 2 - 1) & 1);      // both K tiles' sums are done with it
        if (!ok) break;
#pragma unroll
        for (int k = 0; k < (NQ + 31) / 32; ++k) {
          const int c = lane + 32 * k;
          if (c < NQ) {
            misc->neg_lse[qb][c] = v[k];
            misc->slot[qb][c] = at[k];
          }
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(L_FULL + qb));
      }
    }
  } else if (warp == SUM_WARPS + 2) {
    // =========================== MMA issuer ===========================
    const uint64_t kd0 = ptx::smem_desc_sw128(sbase, 16, 1024);
    const uint64_t qd0 = ptx::smem_desc_sw128(sbase + LY::OFF_Q, 16, 1024);
    const bool lead = ptx::elect_one();
    int kc = 0, qc = 0;
    bool ok = true;
    for (; ok && !walk.done(); walk.next(a, pref)) {
      const Unit x(a, walk);
      if (x.t0 >= x.t1) continue;
      const int kb = kc % LY::KB;
      ok = wait_all(bar(K_FULL + kb), (kc / LY::KB) & 1);
      for (int t = x.t0; t < x.t1 && ok; ++t, ++qc) {
        const int qb = qc & 1, cols = min(QT, x.s.q_len - t * QT) * g_q, n = (cols + STEP - 1) / STEP * STEP;
        const uint32_t idesc = ptx::idesc_bf16_f32(128, 0, false, false) | ((uint32_t)(n >> 3) << 17);
        // (the columns' log-sum-exps as well: who waits for the scores has both)
        ok = wait_all(bar(Q_FULL + qb), (qc / 2) & 1) && wait_all(bar(L_FULL + qb), (qc / 2) & 1);
        for (int s = 0; s < 2 && ok; ++s) {
          if (qc >= 2) ok = wait_all(bar(S_EMPTY + 2 * s + qb), (qc / 2 - 1) & 1);
          if (!ok) break;
          ptx::tc_fence_after();
          if (lead) {
            const uint64_t kd = kd0 + (uint64_t)(((kb * 2 + s) * LY::TILE) >> 4), qd = qd0 + (uint64_t)((qb * LY::Q_TILE) >> 4);
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {
              const uint64_t koff = (uint64_t)(((k >> 2) * (NT * 128) + (k & 3) * 32) >> 4), qoff = (uint64_t)(((k >> 2) * LY::Q_HALF + (k & 3) * 32) >> 4);
              ptx::mma_bf16_ss(tmem + s * 256 + qb * 128, kd + koff, qd + qoff, idesc, k > 0 ? 1u : 0u);
            }
            ptx::mma_commit(bar(S_FULL + 2 * s + qb));
            if (s == 1) {
              ptx::mma_commit(bar(Q_EMPTY + qb));
              if (t == x.t1 - 1) ptx::mma_commit(bar(K_EMPTY + kb));
            }
          }
          __syncwarp();
        }
      }
      ++kc;
    }
    // what has been issued is let run out (bounded) before tensor memory goes back, whoever gave up
    if (lead) ptx::mma_commit(bar(DRAIN));
    for (int k = 0; k < 200000 && !ptx::mbar_try_wait(bar(DRAIN), 0); ++k) {}
    __syncwarp();
  } else if (warp < SUM_WARPS) {
    // =========================== sums ===========================
    const int grp = warp >> 2, s = grp / GROUPS<NQ>, part = grp % GROUPS<NQ>, m = tid & 127;      // K tile, columns' share, row = TMEM lane
    constexpr int SHARE = NQ / GROUPS<NQ>;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + s * 256;
    const float c1 = pd.sm_scale * LOG2E;
    int qc = 0, pieces = 0;
    bool ok = true;
    if (tid == 0) a.cuts[blk].blocks = 0;
    for (; ok && !walk.done(); walk.next(a, pref)) {
      const Unit x(a, walk);
      const int slot = x.slot0 + s * NT + m;
      float total = 0.f, before = 0.f;       // (the old weight is asked for ahead of the waits)
      if (part == 0 && x.whole && slot < x.s.valid) before = old_mass(a, x.b, x.r, slot, x.s);
      const int last_slot = x.slot0 + s * NT + NT - 1;
      for (int t = x.t0; t < x.t1; ++t, ++qc) {
        const int qb = qc & 1, cols = min(QT, x.s.q_len - t * QT) * g_q, n = min((cols + STEP - 1) / STEP * STEP, (part + 1) * SHARE);
        ok = wait_all(bar(S_FULL + 2 * s + qb), (qc / 2) & 1);
        if (!ok) break;
        ptx::tc_fence_after();
        // every column a row that sees every slot of the tile?
        const bool clean = cols >= (part + 1) * SHARE && (long long)x.s.kv - x.s.q_len + t * QT >= last_slot;
        float2 sum[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        const float2 c1v = make_float2(c1, c1);
        const float* nl = misc->neg_lse[qb];
        const int* sl = misc->slot[qb];
        const uint32_t from = lane_addr + qb * 128;
        if (SHARE == 2 * STEP && clean) {      // two loads: the second is on its way while the first is summed
          uint32_t x[STEP], y[STEP];
          ptx::tmem_ld_n<STEP>(x, from + part * SHARE);
          ptx::tmem_wait_ld();
          ptx::tmem_ld_n<STEP>(y, from + part * SHARE + STEP);
          add_columns<STEP, false>(sum, x, c1v, nl + part * SHARE, sl, slot);
          ptx::tmem_wait_ld_regs<STEP>(y);
          add_columns<STEP, false>(sum, y, c1v, nl + part * SHARE + STEP, sl, slot);
        } else {
#pragma unroll 1
          for (int c0 = part * SHARE; c0 < n; c0 += STEP) {
            uint32_t sr[STEP];
            ptx::tmem_ld_n<STEP>(sr, from + c0);
            ptx::tmem_wait_ld();
            add_columns<STEP, true>(sum, sr, c1v, nl + c0, sl + c0, slot);
          }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(S_EMPTY + 2 * s + qb));
        const float2 p = __fadd2_rn(__fadd2_rn(sum[0], sum[1]), __fadd2_rn(sum[2], sum[3]));
        total += p.x + p.y;
      }
      if (!ok) break;
      if constexpr (GROUPS<NQ> == 2) {       // the two shares of the columns meet
        if (part == 1) {
          if (pieces > 0 && !(ok = wait_all(bar(R_EMPTY + s), (pieces - 1) & 1))) break;
          misc->half[s][m] = total;
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(R_FULL + s));
        } else {
          if (!(ok = wait_all(bar(R_FULL + s), pieces & 1))) break;
          total += misc->half[s][m];
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(R_EMPTY + s));
        }
        ++pieces;
      }
      if (part == 0) {
        if (x.whole) {
          if (slot < x.s.valid) a.mass_out[mass_at(a, x.b, x.r, slot)] = total + before;
        } else {
          a.parts[((long long)blk * 2 + (walk.t > 0 ? 0 : 1)) * PAIR + s * NT + m] = total;
          if (tid == 0 && walk.t == 0) {
            MassCut c;                         // up to the block whose range holds the unit's last step
            const long long end = (blk + 1) * all / G - walk.left + walk.n;
            c.blocks = (int)((end * G - 1) / all) - blk + 1;
            c.b = x.b;
            c.r = x.r;
            c.slot0 = x.slot0;
            a.cuts[blk] = c;
          }
        }
      }
    }
    ptx::tc_fence_before();
  }

  __syncthreads();
  if (warp == SUM_WARPS + 2) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, TMEM_COLS);
  }
  if (tid == 0 && misc->abort_flag) report_error(a.sb, DASH_ERR_TIMEOUT, 311);
}

// Adds up the parts of a cut unit: block x the unit that block x of the sums cuts at its end, a thread per slot.
__global__ void __launch_bounds__(PAIR) mass_join_kernel(const __grid_constant__ MassArgs a) {
  chain_wait();
  const int first = blockIdx.x;
  const MassCut c = a.cuts[first];
  if (c.blocks == 0) return;
  float total = a.parts[((long long)first * 2 + 1) * PAIR + threadIdx.x];
#pragma unroll 16
  for (int k = 1; k < c.blocks; ++k) total += a.parts[(long long)(first + k) * 2 * PAIR + threadIdx.x];
  const Seq s = load_seq(a.pd, a.q_start, a.kv_len, c.b);
  const int slot = c.slot0 + threadIdx.x;
  if (slot < s.valid) a.mass_out[mass_at(a, c.b, c.r, slot)] = total + old_mass(a, c.b, c.r, slot, s);
}

template <int HD, int NQ>
cudaError_t launch_one(MassArgs& a, const CUtensorMap& tq, const CUtensorMap& tk, cudaStream_t st) {
  auto kern = key_mass_sm100_kernel<HD, NQ>;
  static std::atomic<unsigned long long> configured{0};
  if (cudaError_t e = allow_dynamic_smem(kern, Layout<HD, NQ>::smem(MAX_SEQS), configured); e != cudaSuccess) return e;
  const int blocks = current_sm_count();
  for (int s0 = 0; s0 < a.pd.batch; s0 += MAX_SEQS) {
    a.seq0 = s0;
    a.n_seqs = a.pd.batch - s0 < MAX_SEQS ? a.pd.batch - s0 : MAX_SEQS;
    cudaError_t e = launch_chained(kern, dim3((unsigned)blocks), dim3(THREADS<NQ>), Layout<HD, NQ>::smem(a.n_seqs), st, tq, tk, a);
    count_launch();
    if (e != cudaSuccess) return e;
    if (a.pd.rows <= a.QT) continue;           // one query tile at most: no unit can be cut
    e = launch_chained(mass_join_kernel, dim3((unsigned)blocks), dim3(PAIR), 0, st, a);
    count_launch();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_key_mass_sm100(const PagedDims& pd, const void* Q, const void* Kpool, const int* page_table, const int* q_start,
                                  const int* kv_len, const float* lse, float decay, const float* mass_in, float* mass_out,
                                  float* partials, StatusBlock* sb, cudaStream_t st) {
  MassArgs a;
  a.pd = pd;
  // Query tiles of 16 columns where the sequences have no more rows than that on average.  16 caches of 8192, 32/8 heads, d 128, tiles of
  // 16 | 128 columns: 1 or 4 tokens each 70 | 72 to 74 us, 5 tokens 78 | 74, 16 tokens 115 | 78.  A prompt among single tokens has the
  // tiles of the average: 255 single tokens and one of 512 over 2048 slots 223 | 266, 63 and one of 190 over 4096 137 | 131.
  const bool few = pd.g_q <= 16 && (long long)pd.rows * pd.g_q <= 16LL * pd.batch;
  a.QT = (few ? 16 : 128) / pd.g_q;
  a.box = paged_box(pd);
  a.q_start = q_start; a.kv_len = kv_len; a.page_table = page_table;
  a.lse = lse; a.mass_in = mass_in; a.mass_out = mass_out;
  a.decay = decay;
  a.cuts = reinterpret_cast<MassCut*>(partials);
  a.parts = partials + (size_t)current_sm_count() * sizeof(MassCut) / sizeof(float);
  a.sb = sb;
  a.inject = test_hooks().skip_own_k_load;
  a.wait_limit = test_hooks().wait_limit_cycles;
  CUtensorMap tq, tk;
  if (!paged_pool_map(&tk, pd, Kpool, pd.ks, a.box)) return cudaErrorInvalidValue;
  PagedDims pq = pd;
  pq.rows = pd.rows > 0 ? pd.rows : 1;       // (a map needs a row; without rows nothing is loaded through it)
  if (!paged_q_map(&tq, pq, pd.rows > 0 ? Q : Kpool, a.QT)) return cudaErrorInvalidValue;
  if (pd.d == 128) return few ? launch_one<128, 16>(a, tq, tk, st) : launch_one<128, 128>(a, tq, tk, st);
  return few ? launch_one<64, 16>(a, tq, tk, st) : launch_one<64, 128>(a, tq, tk, st);
}

}  // namespace dash
