// Shared declarations of the operators around the paged cache (internal; the public ABI is include/dash_attn.h).
#pragma once

#include "common.cuh"

namespace dash {

// Derived problem description handed to kernels by value.
struct PagedDims {
  int batch, rows, h_q, h_kv, d, g_q;
  int dtype;
  int page_size, max_pages, num_pages;
  int cap;             // slots per sequence: max_pages * page_size
  float sm_scale;      // 1 / sqrt(d)
  long long qs[2], kns[2], vns[2], os[2], ks[3], vs[3];
};

// New tokens and cached tokens of one sequence.  Values read from device memory are brought into range here, so that nothing
// indexed with them leaves its buffer, whatever they are.
struct Seq {
  int q0, q_len;    // first packed row, new tokens
  int kv;           // cached tokens as given (at least 0)
  int valid;        // ... that have a slot
};
__device__ __forceinline__ Seq load_seq(const PagedDims& pd, const int* q_start, const int* kv_len, int b) {
  Seq s;
  const int a = __ldg(q_start + b), e = __ldg(q_start + b + 1), kv = __ldg(kv_len + b);
  s.q0 = min(max(a, 0), pd.rows);
  s.q_len = min(max(e, s.q0), pd.rows) - s.q0;
  s.kv = max(kv, 0);
  s.valid = min(s.kv, pd.cap);
  return s;
}

// Last sequence that starts at or before `row` (0 if none does), by a whole warp: 32 probes a round, so that up to 32 sequences
// take one trip to memory and 65535 four.
__device__ __forceinline__ int find_seq(const int* q_start, int batch, int row, int lane) {
  int lo = 0, len = batch;                       // the answer is in [lo, lo + len)
  while (len > 1) {
    const int step = (len + 31) / 32;
    const int probe = lo + lane * step;
    const bool before = lane * step < len && (lane == 0 || __ldg(q_start + probe) <= row);
    const unsigned votes = __ballot_sync(0xffffffffu, before);
    const int hit = 31 - __clz(votes);           // lane 0 always votes
    const int end = lo + len;
    lo += hit * step;
    len = min(step, end - lo);
  }
  return lo;
}

#ifdef __CUDACC__
// 2^x of two values on the FMA pipe, for kernels that the exponential unit would bound (16 a clock and SM): nearest integer by adding
// and taking off 1.5 * 2^23, a polynomial on [-1/2, 1/2], the integer into the exponent bits.  The coefficients are a minimax fit of
// degree 4 with p(0) = 1 (linear program over 2001 points): relative error 2.9e-6.  x below -127 gives exactly 0 (-inf does).
__device__ __forceinline__ float2 exp2_fma(float2 x) {
  const float2 big = make_float2(12582912.f, 12582912.f), nbig = make_float2(-12582912.f, -12582912.f), neg = make_float2(-1.f, -1.f);
  const float2 t = make_float2(fmaxf(x.x, -127.f), fmaxf(x.y, -127.f));
  const float2 r = __fadd2_rn(t, big);
  const float2 f = __ffma2_rn(__fadd2_rn(r, nbig), neg, t);
  float2 p = __ffma2_rn(f, make_float2(0.009581047110259533f, 0.009581047110259533f), make_float2(0.05590597167611122f, 0.05590597167611122f));
  p = __ffma2_rn(f, p, make_float2(0.24024145305156708f, 0.24024145305156708f));
  p = __ffma2_rn(f, p, make_float2(0.6931243538856506f, 0.6931243538856506f));
  p = __ffma2_rn(f, p, make_float2(1.f, 1.f));
  return make_float2(__int_as_float(__float_as_int(p.x) + (__float_as_int(r.x) << 23)),
                     __int_as_float(__float_as_int(p.y) + (__float_as_int(r.y) << 23)));
}
#endif

// Rotary table of a call (kernel argument): frequencies as 64-bit fractions of a turn per position.
constexpr int ROPE_MAX_PAIRS = 64, ROPE_MAX_AXES = 4;
struct RopeTable {
  unsigned long long freq[ROPE_MAX_PAIRS];
  unsigned char axis[ROPE_MAX_PAIRS];
  int pairs;         // 0: no rotation
  int interleaved;
};

cudaError_t launch_rope(const Dims& dm, const RopeTable& rt, const int* positions, const void* Q, const void* K, void* Qout,
                        void* Kout, bool inverse, cudaStream_t st);
cudaError_t launch_append(const PagedDims& pd, const RopeTable& rt, const int* positions, const int* q_start, const int* kv_len,
                          const int* page_table, const void* Q, void* Qout, const void* K, const void* V, void* Kpool,
                          void* Vpool, cudaStream_t st);

bool chunk_sm100_supported(const PagedDims& pd);
size_t chunk_sm100_partial_bytes(const PagedDims& pd);
cudaError_t launch_attend_chunk_sm100(const PagedDims& pd, const void* Q, const void* Kpool, const void* Vpool,
                                      const int* page_table, const int* q_start, const int* kv_len, void* O, float* lse,
                                      float* partials, StatusBlock* sb, cudaStream_t st);
size_t chunk_generic_partial_bytes(const PagedDims& pd);
cudaError_t launch_attend_chunk_generic(const PagedDims& pd, const void* Q, const void* Kpool, const void* Vpool,
                                        const int* page_table, const int* q_start, const int* kv_len, void* O, float* lse,
                                        float* partials, cudaStream_t st);
cudaError_t launch_key_mass_sm100(const PagedDims& pd, const void* Q, const void* Kpool, const int* page_table, const int* q_start,
                                  const int* kv_len, const float* lse, float decay, const float* mass_in, float* mass_out,
                                  float* partials, StatusBlock* sb, cudaStream_t st);
cudaError_t launch_key_mass_generic(const PagedDims& pd, const void* Q, const void* Kpool, const int* page_table,
                                    const int* q_start, const int* kv_len, const float* lse, float decay, const float* mass_in,
                                    float* mass_out, cudaStream_t st);

struct EvictArgs {
  int keep, sinks, recent;
  const float* mass;
  const int* kv_len;
  const int* page_table;
  const char* pool[2];      // K, V
  int* kept;
  int* new_len;
  const int* dst_table;
  int dst_max_pages, dst_num_pages;
  char* dst[2];
  float* mass_out;
  int in_place;
};
cudaError_t launch_evict(const PagedDims& pd, const EvictArgs& a, cudaStream_t st);

}  // namespace dash
