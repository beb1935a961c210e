// Chunk attention and attention weights over a paged cache on CUDA cores (fp32 tensors).
//
// A block takes ROWS (token, head of the group) rows of one (sequence, KV head), token-major, and walks tiles of 64 slots; 256
// threads as 16 x 16, a thread's scores are ROWS / 16 rows by 4 slots, its outputs ROWS / 16 rows by head_dim / 16 columns, both fed
// by 16-byte reads of shared memory (64 FMAs per 8 reads at ROWS = 64).  ROWS = 16 serves calls with few new tokens per sequence,
// where 64 would be mostly empty.  Few units split their slots over blocks (partial m, l, O, joined by a second kernel).
// Tiles come by asynchronous copies behind the arithmetic.  Bound by FFMA issue and the shared-memory reads that feed it.
#include "paged.cuh"

namespace dash {

namespace {

constexpr int KT = 64, THREADS = 256;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct GenArgs {
  PagedDims pd;
  int splits;
  const int *q_start, *kv_len, *page_table;
  const float *Q, *K, *V;
  float *O, *lse, *partials;
  // weights
  const float *lse_in, *mass_in;
  float* mass_out;
  float decay;
};

// Slot t of a sequence's rows: floor(q0 g / ROWS) + b + t (each sequence has as many slots as it has tiles, or more).
__device__ __forceinline__ long long slot_base(const GenArgs& a, int b, int rows_per) {
  const int q0 = min(max(__ldg(a.q_start + b), 0), a.pd.rows);
  return (long long)q0 * a.pd.g_q / rows_per + b;
}

// Asynchronous copies into shared memory, 16 bytes each (src null: zeros; `any` is then a valid address that is not read), in groups.
__device__ __forceinline__ void copy16(float* dst, const float* src, const float* any) {
  const int bytes = src ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((unsigned)__cvta_generic_to_shared(dst)), "l"(src ? src : any), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Where the 64 slots of a tile lie (page, token; page -1: nowhere), worked out by 64 threads a tile ahead and kept in the padding of the K
// rows, two tiles in turn.  (Worked out by every thread for its own copies, a trip to the page table stood before each of them.)
template <int D>
__device__ __forceinline__ int2* where(float* ks, int t, int parity) { return reinterpret_cast<int2*>(ks + t * (D + 4) + D) + parity; }
struct Where {
  int lp, tok, ph;
  __device__ __forceinline__ Where(const PagedDims& pd, const int* table, int slot, int valid) : lp(-1), tok(0), ph(-1) {
    if (slot >= valid) return;
    lp = slot / pd.page_size;
    tok = slot - lp * pd.page_size;
    ph = __ldg(table + lp);
  }
  __device__ __forceinline__ int2 get(const PagedDims& pd) const { return make_int2(ph >= 0 && ph < pd.num_pages ? ph : -1, tok); }
};

// 64 rows of K or V of one (sequence, KV head) into shared memory, row stride LD; slots without a key are zeros.
template <int D, int LD>
__device__ __forceinline__ void load_tile(const PagedDims& pd, const float* pool, const long long* st, int r, float* ks, int parity, float* dst) {
  constexpr int V4 = D / 4;
  pool += r * st[2];
#pragma unroll 4
  for (int k = threadIdx.x; k < KT * V4; k += THREADS) {
    const int t = k / V4, c = k - t * V4;
    const int2 at = *where<D>(ks, t, parity);
    copy16(dst + t * LD + c * 4, at.x >= 0 ? pool + at.x * st[0] + at.y * st[1] + c * 4 : nullptr, pool);
  }
  copies_issued();
}

// Query rows first .. first + ROWS - 1 of the sequence's (token, head) rows; rows behind the last are zeros.
template <int D, int ROWS>
__device__ __forceinline__ void load_rows(const PagedDims& pd, const float* Q, const Seq& s, int r, long long first, float* dst) {
  constexpr int V4 = D / 4;
  const long long n = (long long)s.q_len * pd.g_q;
  for (int k = threadIdx.x; k < ROWS * V4; k += THREADS) {
    const int m = k / V4, c = k - m * V4;
    const long long rho = first + m;
    const float* src = nullptr;
    if (rho < n) {
      const int tok = (int)rho / pd.g_q, hh = (int)rho - tok * pd.g_q;
      src = Q + (long long)(s.q0 + tok) * pd.qs[0] + (long long)(r * pd.g_q + hh) * pd.qs[1] + c * 4;
    }
    copy16(dst + m * D + c * 4, src, Q);
  }
  copies_issued();
}

// acc[i][j] = <row ty * RPT + i, slot tx + 16 j>
template <int D, int RPT>
__device__ __forceinline__ void score_tile(const float* qs, const float* ks, int ty, int tx, float (&acc)[RPT][4]) {
#pragma unroll
  for (int i = 0; i < RPT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
#pragma unroll 4
  for (int c = 0; c < D; c += 4) {
    float4 q[RPT], k[4];
#pragma unroll
    for (int i = 0; i < RPT; ++i) q[i] = *reinterpret_cast<const float4*>(qs + (ty * RPT + i) * D + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const float4*>(ks + (tx + 16 * j) * (D + 4) + c);
#pragma unroll
    for (int i = 0; i < RPT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc[i][j] = fmaf(q[i].x, k[j].x, fmaf(q[i].y, k[j].y, fmaf(q[i].z, k[j].z, fmaf(q[i].w, k[j].w, acc[i][j]))));
  }
}

// Slots that the (token, head) row rho sees.
__device__ __forceinline__ int row_sees(const PagedDims& pd, const Seq& s, long long rho) {
  if (rho >= (long long)s.q_len * pd.g_q) return 0;
  const long long last = (long long)s.kv - s.q_len + rho / pd.g_q + 1;
  return (int)min(max(last, 0LL), (long long)s.valid);
}

// Floats of shared memory: Q, K (rows padded by four), V, P; at D = 128 and 64 rows exactly half of what an SM has.
template <int D, int ROWS> constexpr size_t attend_smem() { return (size_t)(ROWS * D + KT * (D + 4) + KT * D + ROWS * KT) * sizeof(float); }
template <int D, int ROWS> constexpr size_t mass_smem() { return (size_t)(2 * ROWS * D + KT * (D + 4) + 16 * KT) * sizeof(float); }
static_assert(attend_smem<128, 64>() <= 115712 && mass_smem<128, 64>() <= 115712, "two blocks per SM");

template <int D, int ROWS>
__global__ void __launch_bounds__(THREADS, 2) attend_chunk_generic_kernel(const __grid_constant__ GenArgs a) {
  constexpr int RPT = ROWS / 16, CPT = D / 64;        // rows per thread; float4 columns per thread
  constexpr int LDP = KT;
  extern __shared__ float4 smem4[];
  float* qs = reinterpret_cast<float*>(smem4);
  float* ks = qs + ROWS * D;
  float* vs = ks + KT * (D + 4);
  float* ps = vs + KT * D;
  const PagedDims& pd = a.pd;
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int r = (int)(blockIdx.x % pd.h_kv), slot = (int)(blockIdx.x / pd.h_kv), sp = blockIdx.y;
  chain_wait();
  int b = 0;                                  // last sequence whose slots begin at or before this one
  for (int hi = pd.batch; hi - b > 1;) {
    const int mid = (b + hi) >> 1;
    if (slot_base(a, mid, ROWS) <= slot) b = mid; else hi = mid;
  }
  const Seq s = load_seq(pd, a.q_start, a.kv_len, b);
  const long long t = slot - slot_base(a, b, ROWS), first = t * ROWS, n_rows = (long long)s.q_len * pd.g_q;
  if (t < 0 || first >= n_rows) return;
  const int n_tiles = (row_sees(pd, s, min(first + ROWS, n_rows) - 1) + KT - 1) / KT;
  const int t0 = (int)((long long)n_tiles * sp / a.splits), t1 = (int)((long long)n_tiles * (sp + 1) / a.splits);
  const int* table = a.page_table + (long long)b * pd.max_pages;
  load_rows<D, ROWS>(pd, a.Q, s, r, first, qs);
  float m[RPT], l[RPT];
  float4 o[RPT][CPT];
  int sees[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
    sees[i] = row_sees(pd, s, first + ty * RPT + i);
#pragma unroll
    for (int c = 0; c < CPT; ++c) o[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const float c1 = pd.sm_scale * LOG2E;
  // A warp without a row only moves tiles (every warp reads the whole of K and V from shared memory: with one row of sixteen that was
  // what took the time: one token over 36,000 slots, 24/8 heads, d 128, 194 us without this, 96 with it).
  const bool busy = first + (ty & ~1) * RPT < n_rows;
  // K of a tile lands while the product with V of the tile before is formed, V while the scores are
  auto load_k = [&](int j) { load_tile<D, D + 4>(pd, a.K, pd.ks, r, ks, j & 1, ks); };
  auto load_v = [&](int j) { load_tile<D, D>(pd, a.V, pd.vs, r, ks, j & 1, vs); };
  if (tid < 2 * KT) *where<D>(ks, tid & (KT - 1), (t0 + tid / KT) & 1) = Where(pd, table, t0 * KT + tid, s.valid).get(pd);
  __syncthreads();
  if (t0 < t1) {
    load_k(t0);
    load_v(t0);
  }
  for (int j = t0; j < t1; ++j) {
    copies_landed<1>();                                // K (and Q)
    __syncthreads();
    const Where next(pd, table, tid < KT ? (j + 2) * KT + tid : s.valid, s.valid);
    float acc[RPT][4];
    if (busy) score_tile<D, RPT>(qs, ks, ty, tx, acc);
    if (tid < KT) *where<D>(ks, tid, j & 1) = next.get(pd);
    __syncthreads();                                   // K has been read
    if (j + 1 < t1) load_k(j + 1); else copies_issued();
#pragma unroll
    for (int i = 0; i < RPT && busy; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        acc[i][k] = j * KT + tx + 16 * k < sees[i] ? acc[i][k] * c1 : -INFINITY;
        mx = fmaxf(mx, acc[i][k]);
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float mn = fmaxf(m[i], mx), base = mn == -INFINITY ? 0.f : mn;
      const float corr = exp2f(m[i] - base);
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float e = exp2f(acc[i][k] - base);
        sum += e;
        ps[(ty * RPT + i) * LDP + tx + 16 * k] = e;
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
      l[i] = fmaf(l[i], corr, sum);
      m[i] = mn;
#pragma unroll
      for (int c = 0; c < CPT; ++c) {
        o[i][c].x *= corr; o[i][c].y *= corr; o[i][c].z *= corr; o[i][c].w *= corr;
      }
    }
    copies_landed<1>();                                // V
    __syncthreads();
#pragma unroll 2
    for (int k = 0; k < KT && busy; k += 4) {
      float4 p[RPT];
#pragma unroll
      for (int i = 0; i < RPT; ++i) p[i] = *reinterpret_cast<const float4*>(ps + (ty * RPT + i) * LDP + k);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
          const float4 v = *reinterpret_cast<const float4*>(vs + (k + kk) * D + c * 64 + tx * 4);
#pragma unroll
          for (int i = 0; i < RPT; ++i) {
            const float w = kk == 0 ? p[i].x : kk == 1 ? p[i].y : kk == 2 ? p[i].z : p[i].w;
            o[i][c].x = fmaf(w, v.x, o[i][c].x); o[i][c].y = fmaf(w, v.y, o[i][c].y);
            o[i][c].z = fmaf(w, v.z, o[i][c].z); o[i][c].w = fmaf(w, v.w, o[i][c].w);
          }
        }
    }
    __syncthreads();                                   // V and P have been read
    if (j + 1 < t1) load_v(j + 1); else copies_issued();
  }
  copies_landed<0>();
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    if (l[i] != l[i]) m[i] = l[i];            // (a maximum passes over NaN; the row is not to be taken for one without keys)
    const long long rho = first + ty * RPT + i;
    if (rho >= n_rows) continue;
    const int tok = (int)(rho / pd.g_q), hh = (int)(rho - (long long)tok * pd.g_q);
    const long long row = s.q0 + tok, head = r * pd.g_q + hh;
    if (a.splits == 1) {
      const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll
      for (int c = 0; c < CPT; ++c)
        *reinterpret_cast<float4*>(a.O + row * pd.os[0] + head * pd.os[1] + c * 64 + tx * 4) =
            make_float4(o[i][c].x * inv, o[i][c].y * inv, o[i][c].z * inv, o[i][c].w * inv);
      if (tx == 0 && a.lse) a.lse[row * pd.h_q + head] = l[i] == 0.f ? -INFINITY : (m[i] + __log2f(l[i])) * LN2;
    } else {
      float* part = a.partials + (((long long)sp * pd.rows + row) * pd.h_q + head) * (D + 4);
#pragma unroll
      for (int c = 0; c < CPT; ++c) *reinterpret_cast<float4*>(part + c * 64 + tx * 4) = o[i][c];
      if (tx == 0) *reinterpret_cast<float2*>(part + D) = make_float2(m[i], l[i]);
    }
  }
}

// Joins the splits of a row: a warp per (row, head).
template <int D>
__global__ void __launch_bounds__(THREADS) chunk_merge_kernel(const __grid_constant__ GenArgs a) {
  constexpr int VPL = D / 32;
  const PagedDims& pd = a.pd;
  chain_wait();
  const int first = min(max(__ldg(a.q_start), 0), pd.rows), end = min(max(__ldg(a.q_start + pd.batch), first), pd.rows);
  const int lane = threadIdx.x & 31;
  const long long unit = (long long)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5);
  const long long row = unit / pd.h_q, head = unit - row * pd.h_q;
  if (row < first || row >= end) return;
  const long long step = (long long)pd.rows * pd.h_q * (D + 4);
  const float* part = a.partials + unit * (D + 4);
  float mx = -INFINITY;
  for (int k = 0; k < a.splits; ++k) mx = fmaxf(mx, part[k * step + D]);
  float l = 0.f, o[VPL];
#pragma unroll
  for (int c = 0; c < VPL; ++c) o[c] = 0.f;
  for (int k = 0; k < a.splits; ++k) {
    const float2 ml = *reinterpret_cast<const float2*>(part + k * step + D);
    if (ml.x == -INFINITY) continue;
    const float w = exp2f(ml.x - mx);
    l = fmaf(ml.y, w, l);
#pragma unroll
    for (int c = 0; c < VPL; ++c) o[c] = fmaf(part[k * step + c * 32 + lane], w, o[c]);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int c = 0; c < VPL; ++c) a.O[row * pd.os[0] + head * pd.os[1] + c * 32 + lane] = o[c] * inv;
  if (lane == 0 && a.lse) a.lse[unit] = l == 0.f ? -INFINITY : (mx + __log2f(l)) * LN2;
}

// Attention weights per slot: a block keeps a K tile and walks the rows that see it.
template <int D, int ROWS>
__global__ void __launch_bounds__(THREADS, 2) key_mass_generic_kernel(const __grid_constant__ GenArgs a) {
  constexpr int RPT = ROWS / 16;
  extern __shared__ float4 smem4[];
  float* q2 = reinterpret_cast<float*>(smem4);      // two tiles of rows: one lands while the other is read
  float* ks = q2 + 2 * ROWS * D;
  float* red = ks + KT * (D + 4);
  const PagedDims& pd = a.pd;
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int r = blockIdx.y, b = blockIdx.z;
  chain_wait();
  const Seq s = load_seq(pd, a.q_start, a.kv_len, b);
  const long long n_rows = (long long)s.q_len * pd.g_q;
  const int* table = a.page_table + (long long)b * pd.max_pages;
  const float c1 = pd.sm_scale * LOG2E;
  for (int j = blockIdx.x; j * KT < s.valid; j += gridDim.x) {
    __syncthreads();
    if (tid < KT) *where<D>(ks, tid, 0) = Where(pd, table, j * KT + tid, s.valid).get(pd);
    __syncthreads();
    load_tile<D, D + 4>(pd, a.K, pd.ks, r, ks, 0, ks);
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    // the first row that sees the tile's first slot
    const long long i0 = max(0LL, (long long)j * KT - ((long long)s.kv - s.q_len)) * pd.g_q;
    const long long begin = i0 / ROWS * ROWS;
    if (begin < n_rows) load_rows<D, ROWS>(pd, a.Q, s, r, begin, q2);
    int buf = 0;
    for (long long first = begin; first < n_rows; first += ROWS, buf ^= 1) {
      const float* qs = q2 + buf * ROWS * D;
      if (first + ROWS < n_rows) load_rows<D, ROWS>(pd, a.Q, s, r, first + ROWS, q2 + (buf ^ 1) * ROWS * D); else copies_issued();
      copies_landed<1>();
      __syncthreads();
      const bool busy = first + (ty & ~1) * RPT < n_rows;      // (by warps)
      float acc[RPT][4];
      if (busy) score_tile<D, RPT>(qs, ks, ty, tx, acc);
#pragma unroll
      for (int i = 0; i < RPT && busy; ++i) {
        const long long rho = first + ty * RPT + i;
        const int sees = row_sees(pd, s, rho);
        if (sees <= 0) continue;
        const int tok = (int)(rho / pd.g_q), hh = (int)(rho - (long long)tok * pd.g_q);
        const float lse = __ldg(a.lse_in + (long long)(s.q0 + tok) * pd.h_q + r * pd.g_q + hh) * LOG2E;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (j * KT + tx + 16 * k < sees && lse > -INFINITY) sum[k] += exp2f(fmaf(acc[i][k], c1, -lse));
      }
      __syncthreads();                                 // the rows have been read
    }
    copies_landed<0>();
#pragma unroll
    for (int k = 0; k < 4; ++k) red[ty * KT + tx + 16 * k] = sum[k];
    __syncthreads();
    const int slot = j * KT + tid;
    if (tid < KT && slot < s.valid) {
      float total = 0.f;
#pragma unroll
      for (int k = 0; k < 16; ++k) total += red[k * KT + tid];
      const long long at = ((long long)b * pd.h_kv + r) * pd.cap + slot;
      if (a.mass_in && slot < s.kv - s.q_len) total = fmaf(a.decay, a.mass_in[at], total);
      a.mass_out[at] = total;
    }
  }
}

// Rows per tile: 16 where the sequences have fewer than 32 rows on average (64 x 64 tiles would be mostly empty), else 64.  Eight caches
// of 4096, 8/2 heads, d 64, tiles of 16 | 64 rows, attention and weights: 1 token (4 rows) 31 | 35 and 21 | 27 us, 4 tokens 61 | 45 and
// 27 | 29, 7 tokens 81 | 45 and 33 | 31, 8 tokens 80 | 51 and 35 | 31: the weights' line is where it belongs, the attention's would be
// lower, at about 12 rows.  A prompt among single tokens has the tiles of the average: 63 and one of 256 over 2048 slots 148 | 227
// and 233 | 162, 31 and one of 512 (d 128) 442 | 279 and 705 | 252.
int rows_per_tile(const PagedDims& pd) { return (long long)pd.rows * pd.g_q < 32LL * pd.batch ? 16 : 64; }
long long row_slots(const PagedDims& pd) { return (long long)pd.rows * pd.g_q / rows_per_tile(pd) + pd.batch; }

// Splits of the slots: as many blocks as one wave of two per SM takes, pieces of 256 slots at least.  (200 rows over 1500 slots,
// twice, 8/2 heads, d 64: 324 blocks 52 us, 276 blocks 47.)
int generic_splits(const PagedDims& pd) {
  const long long units = row_slots(pd) * pd.h_kv, want = 2LL * current_sm_count() / units;
  const long long most = (pd.cap + 255) / 256;
  return (int)(want < 1 ? 1 : want < most ? (want < 64 ? want : 64) : (most < 64 ? most : 64));
}

template <int D, int ROWS>
cudaError_t launch_attend(GenArgs& a, cudaStream_t st) {
  auto kern = attend_chunk_generic_kernel<D, ROWS>;
  static std::atomic<unsigned long long> configured{0};
  if (cudaError_t e = allow_dynamic_smem(kern, attend_smem<D, ROWS>(), configured); e != cudaSuccess) return e;
  const dim3 grid((unsigned)(row_slots(a.pd) * a.pd.h_kv), (unsigned)a.splits);
  cudaError_t e = launch_chained(kern, grid, dim3(THREADS), attend_smem<D, ROWS>(), st, a);
  count_launch();
  if (e != cudaSuccess || a.splits == 1) return e;
  const long long units = (long long)a.pd.rows * a.pd.h_q;
  e = launch_chained(chunk_merge_kernel<D>, dim3((unsigned)((units + 7) / 8)), dim3(THREADS), 0, st, a);
  count_launch();
  return e;
}

template <int D, int ROWS>
cudaError_t launch_mass(GenArgs& a, cudaStream_t st) {
  auto kern = key_mass_generic_kernel<D, ROWS>;
  static std::atomic<unsigned long long> configured{0};
  if (cudaError_t e = allow_dynamic_smem(kern, mass_smem<D, ROWS>(), configured); e != cudaSuccess) return e;
  const int tiles = (a.pd.cap + KT - 1) / KT;
  cudaError_t e = launch_chained(kern, dim3((unsigned)(tiles < 4096 ? tiles : 4096), (unsigned)a.pd.h_kv, (unsigned)a.pd.batch), dim3(THREADS),
                                 mass_smem<D, ROWS>(), st, a);
  count_launch();
  return e;
}

}  // namespace

size_t chunk_generic_partial_bytes(const PagedDims& pd) {
  const int splits = generic_splits(pd);
  return splits == 1 ? 0 : (size_t)splits * pd.rows * pd.h_q * (pd.d + 4) * sizeof(float);
}

cudaError_t launch_attend_chunk_generic(const PagedDims& pd, const void* Q, const void* Kpool, const void* Vpool,
                                        const int* page_table, const int* q_start, const int* kv_len, void* O, float* lse,
                                        float* partials, cudaStream_t st) {
  GenArgs a = {};
  a.pd = pd;
  a.splits = generic_splits(pd);
  a.q_start = q_start; a.kv_len = kv_len; a.page_table = page_table;
  a.Q = (const float*)Q; a.K = (const float*)Kpool; a.V = (const float*)Vpool;
  a.O = (float*)O; a.lse = lse; a.partials = partials;
  const bool few = rows_per_tile(pd) == 16;
  if (pd.d == 128) return few ? launch_attend<128, 16>(a, st) : launch_attend<128, 64>(a, st);
  return few ? launch_attend<64, 16>(a, st) : launch_attend<64, 64>(a, st);
}

cudaError_t launch_key_mass_generic(const PagedDims& pd, const void* Q, const void* Kpool, const int* page_table,
                                    const int* q_start, const int* kv_len, const float* lse, float decay, const float* mass_in,
                                    float* mass_out, cudaStream_t st) {
  GenArgs a = {};
  a.pd = pd;
  a.q_start = q_start; a.kv_len = kv_len; a.page_table = page_table;
  a.Q = (const float*)Q; a.K = (const float*)Kpool;
  a.lse_in = lse; a.decay = decay; a.mass_in = mass_in; a.mass_out = mass_out;
  const bool few = rows_per_tile(pd) == 16;
  if (pd.d == 128) return few ? launch_mass<128, 16>(a, st) : launch_mass<128, 64>(a, st);
  return few ? launch_mass<64, 16>(a, st) : launch_mass<64, 64>(a, st);
}

}  // namespace dash
