// Attention weight per cached token, summed over a chunk's rows and a group's heads: tensor-core path for sm_100a (bf16).
//
//   mass_t = decay * mass_t + sum over rows (i, h) with slot(i) >= t of exp(s_iht - lse_ih),     s = <q, k_t> / sqrt(d).
// The rows' log-sum-exps are known, so a weight needs no running maximum: the scores are formed transposed, S^T = K Q^T, and a
// thread that owns a slot (a TMEM lane) adds up its row of exponentials.  No exchange between threads, no atomics, one order.
//
// Unit of work: one (sequence, KV head) and 256 slots, two K tiles of 128 that stay in shared memory while the query tiles (NQ
// (token, head) columns) go by; each has a warpgroup and two S buffers in tensor memory, so the MMAs of a tile run while the
// exponentials of the one before are taken.  NQ = 128, or 16 for calls with few new tokens per sequence (decode), which stream K.
// Units are dealt to a persistent grid in turn: neighbours have like costs.
//
// Warp roles (384 threads): warps 0-3, 4-7 sums of the two K tiles; warp 8 loads K (two units deep) and Q tiles; warp 9 the
// log-sum-exps and slots of the columns; warp 10 issues the MMAs.  Every wait is bounded (DASH_ERR_TIMEOUT in the status word).
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
constexpr int THREADS = 384;
constexpr uint32_t TMEM_COLS = 512;          // [K tile][S buffer] of 128 columns
constexpr int MAX_SEQS = 2048;               // sequences of one launch
constexpr float LOG2E = 1.4426950408889634f;

enum Bar { K_FULL = 0, K_EMPTY = 2, Q_FULL = 4, Q_EMPTY = 6, L_FULL = 8, L_EMPTY = 10, S_FULL = 12, S_EMPTY = 16, N_BARS = 20 };

struct Misc {
  unsigned long long bar[N_BARS];
  uint32_t tmem_base;
  int abort_flag;
  __align__(16) float neg_lse[2][128];       // -lse * log2(e) of the columns (-inf: no weight)
  __align__(16) int slot[2][128];            // slots of the columns; -1: no row
  long long scan[THREADS / 32];
};

template <int HD>
struct Layout {
  static constexpr uint32_t TILE = NT * HD * 2;            // regions of 64 elements (128 bytes) per row, 16 KiB apart
  static constexpr uint32_t OFF_Q = 4 * TILE;              // K: [unit parity][tile]
  static constexpr uint32_t OFF_MISC = OFF_Q + 2 * TILE;
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
  StatusBlock* sb;
};

struct Unit {
  int b, r, slot0;                 // first slot
  int t0, t1;                      // query tiles that see it
  Seq s;
};

__device__ __forceinline__ Unit unit_at(const MassArgs& a, const long long* pref, long long u) {
  Unit x;
  int lo = 0, hi = a.n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pref[mid] <= u) lo = mid; else hi = mid;
  }
  x.b = a.seq0 + lo;
  x.s = load_seq(a.pd, a.q_start, a.kv_len, x.b);
  const int per = max(1, (x.s.valid + PAIR - 1) / PAIR);
  const int rest = (int)(u - pref[lo]);
  x.r = rest / per;
  x.slot0 = (rest - x.r * per) * PAIR;
  const long long i0 = max(0LL, (long long)x.slot0 - ((long long)x.s.kv - x.s.q_len));      // first token that sees it
  x.t1 = (x.s.q_len + a.QT - 1) / a.QT;
  x.t0 = (int)min(i0 / a.QT, (long long)x.t1);
  return x;
}

template <int HD, int NQ>
__global__ void __launch_bounds__(THREADS, 1)
key_mass_sm100_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ MassArgs a) {
  using LY = Layout<HD>;
  constexpr int STEP = NQ < 32 ? NQ : 32;    // columns of one tensor-memory load
  extern __shared__ __align__(1024) uint8_t smem[];
  Misc* misc = reinterpret_cast<Misc*>(smem + LY::OFF_MISC);
  long long* pref = reinterpret_cast<long long*>(smem + LY::OFF_PLAN);
  const PagedDims& pd = a.pd;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t sbase = ptx::smem_u32(smem);
  auto bar = [&](int i) { return ptx::smem_u32(&misc->bar[i]); };
  volatile int* abort_flag = &misc->abort_flag;
  auto wait_all = [&](uint32_t barrier, uint32_t parity) { return ptx::mbar_wait_warp(barrier, parity, abort_flag); };
  const int g_q = pd.g_q, QT = a.QT;

  if (tid == 0) {
    misc->abort_flag = (sbase & 1023u) != 0u;
    for (int i = 0; i < N_BARS; ++i)
      ptx::mbar_init(bar(i), i >= S_EMPTY ? 128 : i >= S_FULL ? 1 : i >= L_EMPTY ? 256 : i >= L_FULL ? 32 : 1);
    ptx::fence_barrier_init();
  }
  if (warp == 10) {
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
  // ---- the plan: units of every sequence, summed
  {
    const int per = (a.n_seqs + THREADS - 1) / THREADS, s0 = min(tid * per, a.n_seqs), s1 = min(s0 + per, a.n_seqs);
    long long sum = 0;
    for (int s = s0; s < s1; ++s) {
      const int n = min(max(__ldg(a.kv_len + a.seq0 + s), 0), pd.cap);
      const long long units = (long long)((n + PAIR - 1) / PAIR) * pd.h_kv;
      pref[s] = units;
      sum += units;
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
  const long long units = pref[a.n_seqs];

  if (warp == 8) {
    // =========================== K and Q tiles ===========================
    const int boxes = PAIR / a.box, per_tile = NT / a.box;
    if (lane == 0) {
      ptx::prefetch_tensormap(&tmQ);
      ptx::prefetch_tensormap(&tmK);
    }
    int kc = 0, qc = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
      const Unit x = unit_at(a, pref, u);
      if (x.t0 >= x.t1) continue;
      const int* table = a.page_table + (long long)x.b * pd.max_pages;
      const int slot = x.slot0 + lane * a.box;
      int page = pd.num_pages, tok = 0;      // (out of range: zeros)
      if (lane < boxes && slot < x.s.valid) {
        const int lp = slot / pd.page_size;
        tok = slot - lp * pd.page_size;
        const int ph = __ldg(table + lp);
        if (ph >= 0 && ph < pd.num_pages) page = ph;
      }
      const int kb = kc & 1;
      if (kc >= 2) ok = wait_all(bar(K_EMPTY + kb), (kc / 2 - 1) & 1);
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
            ptx::tma_load_4d(sbase + LY::OFF_Q + qb * LY::TILE + h * (NT * 128), &tmQ, bar(Q_FULL + qb), h * 64, x.r * g_q, x.s.q0 + t * QT, 0);
        }
      }
    }
    if (!ok && lane == 0) {        // let the copies already issued land (bounded) before the block retires
      for (int c = max(0, kc - 2); c < kc; ++c)
        for (int k = 0; k < 200000 && !ptx::mbar_try_wait(bar(K_FULL + (c & 1)), (c / 2) & 1); ++k) {}
      for (int c = max(0, qc - 2); c < qc; ++c)
        for (int k = 0; k < 200000 && !ptx::mbar_try_wait(bar(Q_FULL + (c & 1)), (c / 2) & 1); ++k) {}
    }
  } else if (warp == 9) {
    // =========================== log-sum-exps and slots of the columns ===========================
    int qc = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
      const Unit x = unit_at(a, pref, u);
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
        if (qc >= 2) ok = wait_all(bar(L_EMPTY + qb), (qc / 2 - 1) & 1);
        if (!ok) break;
#pragma unroll
        for (int k = 0; k < (NQ + 31) / 32; ++k) {
          const int c = lane + 32 * k;
          if (c < NQ) {
            misc->neg_lse[qb][c] = v[k];
            misc->slot[qb][c] = at[k];
          }
        }
        ptx::mbar_arrive(bar(L_FULL + qb));
      }
    }
  } else if (warp == 10) {
    // =========================== MMA issuer ===========================
    const uint64_t kd0 = ptx::smem_desc_sw128(sbase, 16, 1024);
    const uint64_t qd0 = ptx::smem_desc_sw128(sbase + LY::OFF_Q, 16, 1024);
    const bool lead = ptx::elect_one();
    int kc = 0, qc = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
      const Unit x = unit_at(a, pref, u);
      if (x.t0 >= x.t1) continue;
      const int kb = kc & 1;
      ok = wait_all(bar(K_FULL + kb), (kc / 2) & 1);
      for (int t = x.t0; t < x.t1 && ok; ++t, ++qc) {
        const int qb = qc & 1, cols = min(QT, x.s.q_len - t * QT) * g_q, n = (cols + STEP - 1) / STEP * STEP;
        const uint32_t idesc = ptx::idesc_bf16_f32(128, 0, false, false) | ((uint32_t)(n >> 3) << 17);
        ok = wait_all(bar(Q_FULL + qb), (qc / 2) & 1);
        for (int s = 0; s < 2 && ok; ++s) {
          if (qc >= 2) ok = wait_all(bar(S_EMPTY + 2 * s + qb), (qc / 2 - 1) & 1);
          if (!ok) break;
          ptx::tc_fence_after();
          if (lead) {
            const uint64_t kd = kd0 + (uint64_t)(((kb * 2 + s) * LY::TILE) >> 4), qd = qd0 + (uint64_t)((qb * LY::TILE) >> 4);
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {
              const uint64_t off = (uint64_t)(((k >> 2) * (NT * 128) + (k & 3) * 32) >> 4);
              ptx::mma_bf16_ss(tmem + s * 256 + qb * 128, kd + off, qd + off, idesc, k > 0 ? 1u : 0u);
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
  } else if (warp < 8) {
    // =========================== sums ===========================
    const int s = warp >> 2, m = tid & 127;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + s * 256;
    const float c1 = pd.sm_scale * LOG2E;
    int qc = 0;
    bool ok = true;
    for (long long u = blockIdx.x; u < units && ok; u += gridDim.x) {
      const Unit x = unit_at(a, pref, u);
      const int slot = x.slot0 + s * NT + m;
      const bool on = slot < x.s.valid;
      const bool old = on && (long long)slot < (long long)x.s.kv - x.s.q_len;
      const long long at = ((long long)x.b * pd.h_kv + x.r) * pd.cap + slot;
      float total = 0.f;
      const float before = old && a.mass_in ? a.mass_in[at] : 0.f;
      const int last_slot = x.slot0 + s * NT + NT - 1;
      for (int t = x.t0; t < x.t1; ++t, ++qc) {
        const int qb = qc & 1, cols = min(QT, x.s.q_len - t * QT) * g_q, n = (cols + STEP - 1) / STEP * STEP;
        const bool here = wait_all(bar(L_FULL + qb), (qc / 2) & 1);
        ok = here && wait_all(bar(S_FULL + 2 * s + qb), (qc / 2) & 1);
        if (!ok) break;
        ptx::tc_fence_after();
        // every column a row that sees every slot of the tile?
        const bool clean = cols == n && (long long)x.s.kv - x.s.q_len + t * QT >= last_slot;
        float2 sum[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        const float2 c1v = make_float2(c1, c1);
#pragma unroll 1
        for (int c0 = 0; c0 < n; c0 += STEP) {
          uint32_t sr[STEP];
          ptx::tmem_ld_n<STEP>(sr, lane_addr + qb * 128 + c0);
          ptx::tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < STEP; c += 4) {
            const float4 nl = *reinterpret_cast<const float4*>(&misc->neg_lse[qb][c0 + c]);
            const float2 e0 = __ffma2_rn(make_float2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])), c1v, make_float2(nl.x, nl.y));
            const float2 e1 = __ffma2_rn(make_float2(__uint_as_float(sr[c + 2]), __uint_as_float(sr[c + 3])), c1v, make_float2(nl.z, nl.w));
            float2 w0 = make_float2(exp2f(e0.x), exp2f(e0.y)), w1 = make_float2(exp2f(e1.x), exp2f(e1.y));
            if (!clean) {
              const int4 sl = *reinterpret_cast<const int4*>(&misc->slot[qb][c0 + c]);
              if (sl.x < slot) w0.x = 0.f;
              if (sl.y < slot) w0.y = 0.f;
              if (sl.z < slot) w1.x = 0.f;
              if (sl.w < slot) w1.y = 0.f;
            }
            sum[(c >> 1) & 2] = __fadd2_rn(sum[(c >> 1) & 2], w0);
            sum[((c >> 1) & 2) + 1] = __fadd2_rn(sum[((c >> 1) & 2) + 1], w1);
          }
        }
        ptx::tc_fence_before();
        ptx::mbar_arrive(bar(S_EMPTY + 2 * s + qb));
        ptx::mbar_arrive(bar(L_EMPTY + qb));
        const float2 p = __fadd2_rn(__fadd2_rn(sum[0], sum[1]), __fadd2_rn(sum[2], sum[3]));
        total += p.x + p.y;
      }
      if (!ok) break;
      if (on) a.mass_out[at] = old ? fmaf(a.decay, before, total) : total;
    }
    ptx::tc_fence_before();
  }

  __syncthreads();
  if (warp == 10) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, TMEM_COLS);
  }
  if (tid == 0 && misc->abort_flag) report_error(a.sb, DASH_ERR_TIMEOUT, 311);
}

template <int HD, int NQ>
cudaError_t launch_one(MassArgs& a, const CUtensorMap& tq, const CUtensorMap& tk, cudaStream_t st) {
  auto kern = key_mass_sm100_kernel<HD, NQ>;
  static std::atomic<unsigned long long> configured{0};
  if (cudaError_t e = allow_dynamic_smem(kern, Layout<HD>::smem(MAX_SEQS), configured); e != cudaSuccess) return e;
  // no more blocks than units that the caches can hold
  const long long most = (long long)a.pd.batch * a.pd.h_kv * ((a.pd.cap + PAIR - 1) / PAIR);
  const int blocks = (int)(most < current_sm_count() ? most : current_sm_count());
  for (int s0 = 0; s0 < a.pd.batch; s0 += MAX_SEQS) {
    a.seq0 = s0;
    a.n_seqs = a.pd.batch - s0 < MAX_SEQS ? a.pd.batch - s0 : MAX_SEQS;
    cudaError_t e = launch_chained(kern, dim3((unsigned)blocks), dim3(THREADS), Layout<HD>::smem(a.n_seqs), st, tq, tk, a);
    count_launch();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_key_mass_sm100(const PagedDims& pd, const void* Q, const void* Kpool, const int* page_table, const int* q_start,
                                  const int* kv_len, const float* lse, float decay, const float* mass_in, float* mass_out,
                                  StatusBlock* sb, cudaStream_t st) {
  MassArgs a;
  a.pd = pd;
  // query tiles of 16 columns where the sequences have no more rows than that on average
  const bool few = pd.g_q <= 16 && (long long)pd.rows * pd.g_q <= 16LL * pd.batch;
  a.QT = (few ? 16 : 128) / pd.g_q;
  a.box = paged_box(pd);
  a.q_start = q_start; a.kv_len = kv_len; a.page_table = page_table;
  a.lse = lse; a.mass_in = mass_in; a.mass_out = mass_out;
  a.decay = decay;
  a.sb = sb;
  CUtensorMap tq, tk;
  if (!paged_pool_map(&tk, pd, Kpool, pd.ks, a.box)) return cudaErrorInvalidValue;
  PagedDims pq = pd;
  pq.rows = pd.rows > 0 ? pd.rows : 1;       // (a map needs a row; without rows nothing is loaded through it)
  if (!paged_q_map(&tq, pq, pd.rows > 0 ? Q : Kpool, a.QT)) return cudaErrorInvalidValue;
  if (pd.d == 128) return few ? launch_one<128, 16>(a, tq, tk, st) : launch_one<128, 128>(a, tq, tk, st);
  return few ? launch_one<64, 16>(a, tq, tk, st) : launch_one<64, 128>(a, tq, tk, st);
}

}  // namespace dash
