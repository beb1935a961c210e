// Rotary positions with several axes, alone (prefill shapes, forward and inverse) and on the way into the paged cache.
//
// Pair i of a head turns by theta = pos[axis(i)] f_i.  In fp32 the product has no fraction left at a far position, so the angle
// is formed in turns as a 64-bit fixed-point fraction: (f_i / 2 pi mod 1) 2^64, multiplied by the position modulo 2^64.  Dropped
// whole turns wrap by themselves and the fraction is exact to the position times 2^-64; its upper 32 bits are kept.  Two more
// bits give the quadrant, the rest lies within an eighth of a turn, where Taylor polynomials (sine to x^9, cosine to x^10)
// are within 2e-9 of the functions.
//
// Memory-bound: every element is read and written once, cosine and sine are formed once per token and pair and serve all heads
// from shared memory.
#include "paged.cuh"

namespace dash {

namespace {

constexpr int THREADS = 256;

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

template <typename T> struct Vec;        // 16 bytes
template <> struct Vec<float> {
  static constexpr int N = 4;
  float v[4];
  __device__ void load(const float* p) { *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(p); }
  __device__ void store(float* p) const { *reinterpret_cast<float4*>(p) = *reinterpret_cast<const float4*>(v); }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  float v[8];
  __device__ void load(const __nv_bfloat16* p) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[k]));
      v[2 * k] = f.x;
      v[2 * k + 1] = f.y;
    }
  }
  __device__ void store(__nv_bfloat16* p) const {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
      w[k] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// One head's row: `items` pieces of work, piece `v` reads and writes two vectors (or, SCALAR, two elements) of it.
//   halves       vectors v and pairs / N + v hold the two sides of N pairs; behind the pairs two vectors pass through
//   interleaved  a vector holds N / 2 whole pairs
// SCALAR serves pair counts that are no multiple of a vector: element pairs, one at a time.
template <typename T, bool SCALAR>
__device__ __forceinline__ void turn_piece(const T* src, T* dst, int v, int d, int pairs, bool interleaved, const float2* cs) {
  constexpr int N = Vec<T>::N;
  if constexpr (SCALAR) {
    int lo = 2 * v, hi = 2 * v + 1;             // behind the pairs (2 v >= 2 pairs) and interleaved: neighbours
    if (v < pairs && !interleaved) { lo = v; hi = v + pairs; }
    const float x = to_f32(src[lo]), y = to_f32(src[hi]);
    const float2 t = v < pairs ? cs[v] : make_float2(1.f, 0.f);
    dst[lo] = from_f32<T>(fmaf(x, t.x, -(y * t.y)));
    dst[hi] = from_f32<T>(fmaf(x, t.y, y * t.x));
  } else {
    const int per = pairs / N;                  // pieces that hold pairs by halves
    const bool turn = interleaved ? 2 * v * N < 2 * pairs : v < per;
    const int lo = interleaved || !turn ? 2 * v * N : v * N;
    const int hi = interleaved || !turn ? lo + N : pairs + v * N;
    Vec<T> a, b;
    a.load(src + lo);
    b.load(src + hi);
    if (turn) {
      if (interleaved) {
#pragma unroll
        for (int k = 0; k < N; k += 2) {
          const float2 t = cs[(lo + k) >> 1];
          const float x = a.v[k], y = a.v[k + 1];
          a.v[k] = fmaf(x, t.x, -(y * t.y));
          a.v[k + 1] = fmaf(x, t.y, y * t.x);
        }
        if (hi < 2 * pairs) {
#pragma unroll
          for (int k = 0; k < N; k += 2) {
            const float2 t = cs[(hi + k) >> 1];
            const float x = b.v[k], y = b.v[k + 1];
            b.v[k] = fmaf(x, t.x, -(y * t.y));
            b.v[k + 1] = fmaf(x, t.y, y * t.x);
          }
        }
      } else {
        const float4* t4 = reinterpret_cast<const float4*>(cs + lo);
#pragma unroll
        for (int k = 0; k < N; k += 2) {
          const float4 t = t4[k >> 1];
          float x = a.v[k], y = b.v[k];
          a.v[k] = fmaf(x, t.x, -(y * t.y));
          b.v[k] = fmaf(x, t.y, y * t.x);
          x = a.v[k + 1], y = b.v[k + 1];
          a.v[k + 1] = fmaf(x, t.z, -(y * t.w));
          b.v[k + 1] = fmaf(x, t.w, y * t.z);
        }
      }
    }
    a.store(dst + lo);
    b.store(dst + hi);
  }
}

// Cosines and sines of the block's tokens: cs[token][pair].  `at(token)` = base index into positions, or < 0 for no such token.
template <typename At>
__device__ __forceinline__ void fill_table(float2* cs, const RopeTable& rt, const int* positions, long long axis_stride, int tokens,
                                           float sign, At&& at) {
  for (int k = threadIdx.x; k < tokens * rt.pairs; k += THREADS) {
    const int t = k / rt.pairs, i = k - t * rt.pairs;
    const long long base = at(t);
    if (base < 0) continue;
    float2 c = cos_sin_of_turns(rt.freq[i], __ldg(positions + (long long)rt.axis[i] * axis_stride + base));
    c.y *= sign;
    cs[k] = c;
  }
}

struct RopeArgs {
  RopeTable rt;
  const void *Q, *K;
  void *Qout, *Kout;
  const int* positions;
  long long qs[3], ks[3];
  int batch, n, h_q, h_k, d, tokens;    // h_q / h_k: 0 where the tensor is absent; tokens per block
  float sign;
};

template <typename T, bool SCALAR>
__global__ void __launch_bounds__(THREADS) rope_kernel(const __grid_constant__ RopeArgs a) {
  extern __shared__ float4 cs4[];
  float2* cs = reinterpret_cast<float2*>(cs4);
  chain_wait();
  const long long total = (long long)a.batch * a.n, first = (long long)blockIdx.x * a.tokens;
  const int here = (int)min((long long)a.tokens, total - first);
  fill_table(cs, a.rt, a.positions, total, here, a.sign, [&](int t) { return first + t; });
  __syncthreads();
  const int per_head = a.d / (SCALAR ? 2 : 2 * Vec<T>::N), heads = a.h_q + a.h_k, per_token = heads * per_head;
#pragma unroll 2
  for (int k = threadIdx.x; k < here * per_token; k += THREADS) {
    const int t = k / per_token, rem = k - t * per_token;
    const int h = rem / per_head, v = rem - h * per_head;
    const long long b = (first + t) / a.n, i = (first + t) - b * a.n;
    const bool q = h < a.h_q;
    const long long off = q ? b * a.qs[0] + i * a.qs[1] + h * a.qs[2] : b * a.ks[0] + i * a.ks[1] + (h - a.h_q) * a.ks[2];
    turn_piece<T, SCALAR>((const T*)(q ? a.Q : a.K) + off, (T*)(q ? a.Qout : a.Kout) + off, v, a.d, a.rt.pairs,
                          a.rt.interleaved != 0, cs + t * a.rt.pairs);
  }
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

constexpr int APPEND_TOKENS = 8;

template <typename T, bool SCALAR>
__global__ void __launch_bounds__(THREADS) append_kernel(const __grid_constant__ AppendArgs a) {
  extern __shared__ float4 cs4[];
  float2* cs = reinterpret_cast<float2*>(cs4);
  __shared__ long long page_of[APPEND_TOKENS];    // physical page, -1: no slot, -2: not a row of any sequence
  __shared__ int tok_of[APPEND_TOKENS];
  const PagedDims& pd = a.pd;
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
  if (a.rt.pairs) fill_table(cs, a.rt, a.positions, pd.rows, here, 1.f, [&](int t) { return (long long)first + t; });
  __syncthreads();
  const int per_head = pd.d / (SCALAR ? 2 : 2 * Vec<T>::N), heads = a.h_q + 2 * pd.h_kv, per_token = heads * per_head;
#pragma unroll 2
  for (int k = threadIdx.x; k < here * per_token; k += THREADS) {
    const int t = k / per_token, rem = k - t * per_token;
    int h = rem / per_head;
    const int v = rem - h * per_head, tok = tok_of[t];
    const long long row = first + t, page = page_of[t];
    const T* src;
    T* dst;
    int pairs = a.rt.pairs;
    if (h < a.h_q) {
      if (page == -2) continue;
      src = (const T*)a.Q + row * pd.qs[0] + h * pd.qs[1];
      dst = (T*)a.Qout + row * pd.os[0] + h * pd.os[1];
    } else {
      if (page < 0) continue;
      h -= a.h_q;
      if (h < pd.h_kv) {
        src = (const T*)a.K + row * pd.kns[0] + h * pd.kns[1];
        dst = (T*)a.Kpool + page * pd.ks[0] + tok * pd.ks[1] + h * pd.ks[2];
      } else {
        h -= pd.h_kv;
        src = (const T*)a.V + row * pd.vns[0] + h * pd.vns[1];
        dst = (T*)a.Vpool + page * pd.vs[0] + tok * pd.vs[1] + h * pd.vs[2];
        pairs = 0;
      }
    }
    turn_piece<T, SCALAR>(src, dst, v, pd.d, pairs, a.rt.interleaved != 0, cs + t * a.rt.pairs);
  }
}

// Whole vectors where every side of the pairs is made of them: by halves the pairs, interleaved the pairs' elements, have to be a
// multiple of a vector, and what passes through a multiple of two.
bool by_vectors(const RopeTable& rt, int d, int n) {
  if (rt.interleaved) return (2 * rt.pairs) % n == 0;
  return rt.pairs % n == 0 && (d - 2 * rt.pairs) % (2 * n) == 0;
}

// Tokens per block: one where the blocks would not fill the machine otherwise, eight where they do (a block's table is then formed
// by all of its threads).
int tokens_per_block(long long tokens) { return tokens >= 8LL * 4 * current_sm_count() ? 8 : tokens >= 4LL * current_sm_count() ? 2 : 1; }

template <typename T>
cudaError_t launch_rope_t(RopeArgs& a, cudaStream_t st) {
  const long long total = (long long)a.batch * a.n;
  a.tokens = tokens_per_block(total);
  const unsigned blocks = (unsigned)((total + a.tokens - 1) / a.tokens);
  const size_t smem = (size_t)a.tokens * a.rt.pairs * sizeof(float2);
  const bool vec = by_vectors(a.rt, a.d, Vec<T>::N);
  cudaError_t e = launch_chained(vec ? rope_kernel<T, false> : rope_kernel<T, true>, dim3(blocks), dim3(THREADS), smem, st, a);
  count_launch();
  return e;
}

template <typename T>
cudaError_t launch_append_t(AppendArgs& a, cudaStream_t st) {
  a.tokens = tokens_per_block(a.pd.rows);
  const unsigned blocks = (unsigned)((a.pd.rows + a.tokens - 1) / a.tokens);
  const size_t smem = (size_t)a.tokens * a.rt.pairs * sizeof(float2);
  const bool vec = by_vectors(a.rt, a.pd.d, Vec<T>::N);
  cudaError_t e = launch_chained(vec ? append_kernel<T, false> : append_kernel<T, true>, dim3(blocks), dim3(THREADS), smem, st, a);
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
