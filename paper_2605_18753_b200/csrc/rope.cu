// Rotary positions with several axes, alone (prefill shapes, forward and inverse) and on the way into the paged cache.
//
// Pair i of a head turns by theta = pos[axis(i)] f_i.  In fp32 the product has no fraction left at a far position, so the angle
// is formed in turns as a 64-bit fixed-point fraction: (f_i / 2 pi mod 1) 2^64, multiplied by the position modulo 2^64.  Dropped
// whole turns wrap by themselves and the fraction is exact to the position times 2^-64; its upper 32 bits are kept (2^-31 turns in
// all).  Two more bits give the quadrant, the rest lies within an eighth of a turn, where Taylor polynomials (sine to x^9, cosine
// to x^10) are within 2e-9 of the functions.
//
// Memory-bound: every element is read and written once.  A thread owns one piece of the head (N pairs: two 16-byte vectors) of one
// token, forms its cosines and sines in registers and takes the piece through its share of the heads, four heads on their way
// at once; the eight lanes of a head cover whole lines.  8192 tokens, 40 heads, d 128: 29.8 us (5.6 TB/s, 86 % of the measured copy);
// with a table in shared memory for all heads of a token 42 (bank conflicts, a barrier), one head on its way at a time 45, eight 34,
// four with the next four behind them 35 to 44.  12,300 tokens with their K and V into pages: 39.3 us (5.3 TB/s);
// 4500 in fp32 45.1 us (4.9 TB/s, cold).  Pair counts that are no multiple of a vector go element by element: the 8192 tokens above 49
// to 51 us cold where vectors take 37, in fp32 62 to 66 where they take 60 to 66.
// Small blocks: each goes through phases (loads, cosines, stores), and the more of them share an SM the better the phases mix; of 64, 128
// and 256 threads at the same number of threads per SM 29.8 / 30.7 / 32.3 us, and 39.3 / 39.8 / 44.6 into pages.
#include <type_traits>

#include "paged.cuh"

namespace dash {

namespace {

constexpr int THREADS = 64;
constexpr int ROPE_TOKENS = 2, APPEND_TOKENS = 4;      // per block, at most (4 and 2: 32.7 us alone, 40.8 into pages)

__device__ __forceinline__ float2 cos_sin_of_turns(unsigned long long freq, int pos) {
  const unsigned long long turns = freq * (unsigned long long)(long long)pos;
  const unsigned int frac = (unsigned int)(turns >> 32);
  const unsigned int q = (frac + 0x20000000u) >> 30;                        // nearest quarter turn
  const float a = (float)(int)(frac - (q << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float z = a * a;
  float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  s = fmaf(z, s, 8.3333333e-3f);
  s = fmaf(z, s, -1.6666667e-1f);
  s = fmaf(a * z, s, a);
  float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(z, c, -1.3888889e-3f);
  c = fmaf(z, c, 4.1666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.f);
  float2 r = (q & 1) ? make_float2(-s, c) : make_float2(c, s);
  if (q & 2) r = make_float2(-r.x, -r.y);
  return r;
}

// 16 bytes, as they lie in memory until they are needed.
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  float4 raw;
  __device__ void load(const float* p) { raw = *reinterpret_cast<const float4*>(p); }
  __device__ void get(float (&v)[4]) const { v[0] = raw.x; v[1] = raw.y; v[2] = raw.z; v[3] = raw.w; }
  static __device__ void store(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  uint4 raw;
  __device__ void load(const __nv_bfloat16* p) { raw = *reinterpret_cast<const uint4*>(p); }
  __device__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[k]));
      v[2 * k] = f.x;
      v[2 * k + 1] = f.y;
    }
  }
  static __device__ void store(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
      w[k] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// A piece of a head: piece v has pairs v N .. v N + N - 1 (SCALAR: pair v alone).
//   halves       the pairs' first elements are one vector, their second elements another
//   interleaved  the pairs fill two vectors one behind the other
// Behind the rotated pairs both are two neighbouring vectors (elements) that pass through.  SCALAR serves pair counts that are no
// multiple of a vector.
template <typename T, bool SCALAR, bool IL>
struct Piece {
  static constexpr int N = SCALAR ? 1 : Vec<T>::N;
  float2 cs[N];
  int lo, hi;
  bool turn_lo, turn_hi;                       // (interleaved: the two vectors apart; halves: both)
  __device__ __forceinline__ void place(const RopeTable& rt, int v) {
    const int first = v * N;
    turn_lo = first < rt.pairs;
    turn_hi = IL && !SCALAR ? first + N / 2 < rt.pairs : turn_lo;
    lo = IL || !turn_lo ? 2 * first : first;
    hi = IL || !turn_lo ? 2 * first + N : first + rt.pairs;
  }
  // pos(axis): the token's position
  template <typename Pos>
  __device__ __forceinline__ void prepare(const RopeTable& rt, int v, float sign, Pos&& pos) {
    const int first = v * N;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      cs[k] = make_float2(1.f, 0.f);
      if (first + k < rt.pairs) {
        cs[k] = cos_sin_of_turns(rt.freq[first + k], pos(rt.axis[first + k]));
        cs[k].y *= sign;
      }
    }
  }
  static __device__ __forceinline__ void turn(float& x, float& y, float2 t) {
    const float a = x, b = y;
    x = fmaf(a, t.x, -(b * t.y));
    y = fmaf(a, t.y, b * t.x);
  }
  using Side = std::conditional_t<SCALAR, T, Vec<T>>;
  __device__ __forceinline__ void load(const T* src, Side& a, Side& b) const {
    if constexpr (SCALAR) {
      a = src[lo];
      b = src[hi];
    } else {
      a.load(src + lo);
      b.load(src + hi);
    }
  }
  __device__ __forceinline__ void finish(T* dst, const Side& a, const Side& b, bool rotate) const {
    if constexpr (SCALAR) {
      float x = to_f32(a), y = to_f32(b);
      if (rotate && turn_lo) turn(x, y, cs[0]);
      dst[lo] = from_f32<T>(x);
      dst[hi] = from_f32<T>(y);
    } else {
      float x[N], y[N];
      a.get(x);
      b.get(y);
      if (rotate) {
        if constexpr (IL) {
          if (turn_lo) {
#pragma unroll
            for (int k = 0; k < N; k += 2) turn(x[k], x[k + 1], cs[k / 2]);
          }
          if (turn_hi) {
#pragma unroll
            for (int k = 0; k < N; k += 2) turn(y[k], y[k + 1], cs[N / 2 + k / 2]);
          }
        } else if (turn_lo) {
#pragma unroll
          for (int k = 0; k < N; ++k) turn(x[k], y[k], cs[k]);
        }
      }
      Vec<T>::store(dst + lo, x);
      Vec<T>::store(dst + hi, y);
    }
  }
  // The piece of BATCH heads from h on, `step` apart, on its way at once: the output may be the input, so the compiler would finish one
  // head before it asks for the next.
  static constexpr int BATCH = 4;
  struct Heads { Side a[BATCH], b[BATCH]; };
  __device__ __forceinline__ void fetch(Heads& x, const T* src, long long stride, int h, int step, int heads) const {
#pragma unroll
    for (int k = 0; k < BATCH; ++k)
      if (h + k * step < heads) load(src + (h + k * step) * stride, x.a[k], x.b[k]);
  }
  __device__ __forceinline__ void finish(const Heads& x, T* dst, long long stride, int h, int step, int heads, bool rotate) const {
#pragma unroll
    for (int k = 0; k < BATCH; ++k)
      if (h + k * step < heads) finish(dst + (h + k * step) * stride, x.a[k], x.b[k], rotate);
  }
  // Heads first, first + step, ... below `heads`; x: the first batch, fetched.
  __device__ __forceinline__ void run(Heads& x, const T* src, T* dst, long long src_stride, long long dst_stride, int first, int step, int heads,
                                      bool rotate) const {
    for (int h = first; h < heads; h += BATCH * step) {
      if (h != first) fetch(x, src, src_stride, h, step, heads);
      finish(x, dst, dst_stride, h, step, heads, rotate);
    }
  }
};

// A block: `tokens` tokens, `pieces` threads per head, and what is left of its threads as groups that share the heads.
struct Share {
  int v, t, group, groups;
  __device__ __forceinline__ Share(int pieces, int tokens) {
    const int log_p = 31 - __clz(pieces), rest = (int)threadIdx.x >> log_p, log_t = 31 - __clz(tokens);      // (powers of two)
    v = threadIdx.x & (pieces - 1);
    t = rest & (tokens - 1);
    group = rest >> log_t;
    groups = THREADS >> (log_p + log_t);
  }
};

struct RopeArgs {
  RopeTable rt;
  const void *Q, *K;
  void *Qout, *Kout;
  const int* positions;
  long long qs[3], ks[3];
  int batch, n, h_q, h_k, d, tokens;    // h_q / h_k: 0 where the tensor is absent; tokens per block
  float sign;
};

template <typename T, bool SCALAR, bool IL>
__global__ void __launch_bounds__(THREADS, 10) rope_kernel(const __grid_constant__ RopeArgs a) {
  using P = Piece<T, SCALAR, IL>;
  const Share sh(a.d / (2 * P::N), a.tokens);
  chain_wait();
  const long long total = (long long)a.batch * a.n, token = (long long)blockIdx.x * a.tokens + sh.t;
  if (token >= total) return;
  P p;
  typename P::Heads x;
  p.place(a.rt, sh.v);
  const long long b = token / a.n, i = token - b * a.n;
  const long long qo = b * a.qs[0] + i * a.qs[1], ko = b * a.ks[0] + i * a.ks[1];
  p.fetch(x, (const T*)a.Q + qo, a.qs[2], sh.group, sh.groups, a.h_q);
  p.prepare(a.rt, sh.v, a.sign, [&](int axis) { return __ldg(a.positions + axis * total + token); });
  p.run(x, (const T*)a.Q + qo, (T*)a.Qout + qo, a.qs[2], a.qs[2], sh.group, sh.groups, a.h_q, true);
  p.fetch(x, (const T*)a.K + ko, a.ks[2], sh.group, sh.groups, a.h_k);
  p.run(x, (const T*)a.K + ko, (T*)a.Kout + ko, a.ks[2], a.ks[2], sh.group, sh.groups, a.h_k, true);
}

struct AppendArgs {
  RopeTable rt;
  PagedDims pd;
  const int *positions, *q_start, *kv_len, *page_table;
  const void *Q, *K, *V;
  void *Qout, *Kpool, *Vpool;
  int h_q;        // 0: no queries
  int tokens;     // per block
};


template <typename T, bool SCALAR, bool IL>
__global__ void __launch_bounds__(THREADS, 8) append_kernel(const __grid_constant__ AppendArgs a) {
  using P = Piece<T, SCALAR, IL>;
  __shared__ long long page_of[APPEND_TOKENS];    // physical page, -1: no slot, -2: not a row of any sequence
  __shared__ int tok_of[APPEND_TOKENS];
  const PagedDims& pd = a.pd;
  const Share sh(pd.d / (2 * P::N), a.tokens);
  chain_wait();
  const int first = blockIdx.x * a.tokens, here = min(a.tokens, pd.rows - first);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int t = warp; t < here; t += THREADS / 32) {
    const int row = first + t, b = find_seq(a.q_start, pd.batch, row, lane);
    const Seq s = load_seq(pd, a.q_start, a.kv_len, b);
    long long page = -2;
    int tok = 0;
    if (row >= s.q0 && row < s.q0 + s.q_len) {
      const int slot = s.kv - s.q_len + (row - s.q0);
      page = -1;
      if (slot >= 0 && slot < pd.cap) {
        const int lp = slot / pd.page_size;
        tok = slot - lp * pd.page_size;
        const int ph = __ldg(a.page_table + (long long)b * pd.max_pages + lp);
        if (ph >= 0 && ph < pd.num_pages) page = ph;
      }
    }
    if (lane == 0) {
      page_of[t] = page;
      tok_of[t] = tok;
    }
  }
  P p;
  typename P::Heads x;
  p.place(a.rt, sh.v);
  const long long row = first + sh.t;
  const bool rotate = a.rt.pairs > 0;
  const T *q = (const T*)a.Q + row * pd.qs[0], *k = (const T*)a.K + row * pd.kns[0], *v = (const T*)a.V + row * pd.vns[0];
  if (sh.t < here) p.fetch(x, q, pd.qs[1], sh.group, sh.groups, a.h_q);
  p.prepare(a.rt, sh.v, 1.f, [&](int axis) { return sh.t < here ? __ldg(a.positions + (long long)axis * pd.rows + row) : 0; });
  __syncthreads();
  if (sh.t >= here) return;
  const long long page = page_of[sh.t];
  const int tok = tok_of[sh.t];
  if (page == -2) return;
  p.run(x, q, (T*)a.Qout + row * pd.os[0], pd.qs[1], pd.os[1], sh.group, sh.groups, a.h_q, rotate);
  if (page < 0) return;
  p.fetch(x, k, pd.kns[1], sh.group, sh.groups, pd.h_kv);
  typename P::Heads y;
  p.fetch(y, v, pd.vns[1], sh.group, sh.groups, pd.h_kv);
  p.run(x, k, (T*)a.Kpool + page * pd.ks[0] + tok * pd.ks[1], pd.kns[1], pd.ks[2], sh.group, sh.groups, pd.h_kv, rotate);
  p.run(y, v, (T*)a.Vpool + page * pd.vs[0] + tok * pd.vs[1], pd.vns[1], pd.vs[2], sh.group, sh.groups, pd.h_kv, false);
}

// Whole vectors where every side of the pairs is made of them: by halves the pairs, interleaved the pairs' elements, have to be a
// multiple of a vector, and what passes through a multiple of two.
bool by_vectors(const RopeTable& rt, int d, int n) {
  if (rt.interleaved) return (2 * rt.pairs) % n == 0;
  return rt.pairs % n == 0 && (d - 2 * rt.pairs) % (2 * n) == 0;
}

// Tokens per block: `most` where there are many (the cosines of a piece serve more heads), fewer where that would leave the machine
// short of blocks (eight per SM; a token's heads are then shared by more threads).
int tokens_per_block(long long tokens, int pieces, int most) {
  int t = most;
  while (t > 1 && (t * pieces > THREADS || tokens < 8LL * t * current_sm_count())) t >>= 1;
  return t;
}

template <typename T>
cudaError_t launch_rope_t(RopeArgs& a, cudaStream_t st) {
  const long long total = (long long)a.batch * a.n;
  const bool vec = by_vectors(a.rt, a.d, Vec<T>::N);
  a.tokens = tokens_per_block(total, a.d / (vec ? 2 * Vec<T>::N : 2), ROPE_TOKENS);
  const unsigned blocks = (unsigned)((total + a.tokens - 1) / a.tokens);
  auto kern = vec ? (a.rt.interleaved ? rope_kernel<T, false, true> : rope_kernel<T, false, false>)
                  : (a.rt.interleaved ? rope_kernel<T, true, true> : rope_kernel<T, true, false>);
  cudaError_t e = launch_chained(kern, dim3(blocks), dim3(THREADS), 0, st, a);
  count_launch();
  return e;
}

template <typename T>
cudaError_t launch_append_t(AppendArgs& a, cudaStream_t st) {
  const bool vec = by_vectors(a.rt, a.pd.d, Vec<T>::N);
  a.tokens = tokens_per_block(a.pd.rows, a.pd.d / (vec ? 2 * Vec<T>::N : 2), APPEND_TOKENS);
  const unsigned blocks = (unsigned)((a.pd.rows + a.tokens - 1) / a.tokens);
  auto kern = vec ? (a.rt.interleaved ? append_kernel<T, false, true> : append_kernel<T, false, false>)
                  : (a.rt.interleaved ? append_kernel<T, true, true> : append_kernel<T, true, false>);
  cudaError_t e = launch_chained(kern, dim3(blocks), dim3(THREADS), 0, st, a);
  count_launch();
  return e;
}

}  // namespace

cudaError_t launch_rope(const Dims& dm, const RopeTable& rt, const int* positions, const void* Q, const void* K, void* Qout,
                        void* Kout, bool inverse, cudaStream_t st) {
  RopeArgs a;
  a.rt = rt;
  a.Q = Q; a.K = K; a.Qout = Qout; a.Kout = Kout;
  a.positions = positions;
  for (int k = 0; k < 3; ++k) { a.qs[k] = dm.qs[k]; a.ks[k] = dm.ks[k]; }
  a.batch = dm.batch; a.n = dm.seq_q; a.h_q = Q ? dm.h_q : 0; a.h_k = K ? dm.h_kv : 0; a.d = dm.d;
  a.sign = inverse ? -1.f : 1.f;
  return dm.dtype == DASH_BF16 ? launch_rope_t<__nv_bfloat16>(a, st) : launch_rope_t<float>(a, st);
}

cudaError_t launch_append(const PagedDims& pd, const RopeTable& rt, const int* positions, const int* q_start, const int* kv_len,
                          const int* page_table, const void* Q, void* Qout, const void* K, const void* V, void* Kpool,
                          void* Vpool, cudaStream_t st) {
  AppendArgs a;
  a.rt = rt; a.pd = pd;
  a.positions = positions; a.q_start = q_start; a.kv_len = kv_len; a.page_table = page_table;
  a.Q = Q; a.K = K; a.V = V; a.Qout = Qout; a.Kpool = Kpool; a.Vpool = Vpool;
  a.h_q = Q ? pd.h_q : 0;
  return pd.dtype == DASH_BF16 ? launch_append_t<__nv_bfloat16>(a, st) : launch_append_t<float>(a, st);
}

}  // namespace dash
