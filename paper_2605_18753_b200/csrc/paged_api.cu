// C ABI of the operators around the paged cache: argument validation and dispatch.  Every operation is defined in
// include/dash_attn.h; kernels live in rope.cu, chunk_sm100.cu, chunk_generic.cu, key_mass_sm100.cu and evict.cu.
#include <cmath>
#include <cstring>

#include <nvtx3/nvToolsExt.h>

#include "paged.cuh"

namespace dash {

namespace {

struct StageRange {
  explicit StageRange(const char* name) { nvtxRangePushA(name); }
  ~StageRange() { nvtxRangePop(); }
};

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
int cuda_status(cudaError_t e) { return e == cudaSuccess ? DASH_OK : DASH_ERR_CUDA; }

template <int N>
bool good_strides(const int64_t* s, int dtype, long long* out) {
  const int mult = dtype == DASH_BF16 ? 8 : 4;
  for (int k = 0; k < N; ++k) {
    if (s[k] < 0 || s[k] % mult != 0 || s[k] > ((long long)1 << 40)) return false;
    out[k] = s[k];
  }
  return true;
}

int make_paged(const dash_paged_params* p, PagedDims* pd) {
  if (!p || p->struct_size != sizeof(dash_paged_params)) return DASH_ERR_INVALID_ARG;
  if (p->batch <= 0 || p->batch > 65535 || p->rows < 0 || p->h_q <= 0 || p->h_kv <= 0 || p->h_kv > 65535) return DASH_ERR_INVALID_ARG;
  if (p->h_q % p->h_kv != 0) return DASH_ERR_INVALID_ARG;
  if (p->dtype != DASH_F32 && p->dtype != DASH_BF16) return DASH_ERR_INVALID_ARG;
  if (p->page_size <= 0 || p->page_size % 16 != 0 || p->max_pages <= 0 || p->num_pages <= 0) return DASH_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return DASH_ERR_UNSUPPORTED;
  if (p->h_q / p->h_kv > 128) return DASH_ERR_UNSUPPORTED;
  if ((long long)p->max_pages * p->page_size > (1 << 25)) return DASH_ERR_UNSUPPORTED;
  if ((long long)p->rows * p->h_q > 0x7fffffffLL || (long long)p->batch * p->h_kv > (1 << 24)) return DASH_ERR_UNSUPPORTED;
  std::memset(pd, 0, sizeof(*pd));
  if (!good_strides<2>(p->q_stride, p->dtype, pd->qs) || !good_strides<2>(p->kn_stride, p->dtype, pd->kns) ||
      !good_strides<2>(p->vn_stride, p->dtype, pd->vns) || !good_strides<2>(p->o_stride, p->dtype, pd->os) ||
      !good_strides<3>(p->k_stride, p->dtype, pd->ks) || !good_strides<3>(p->v_stride, p->dtype, pd->vs))
    return DASH_ERR_INVALID_ARG;
  pd->batch = p->batch; pd->rows = p->rows; pd->h_q = p->h_q; pd->h_kv = p->h_kv; pd->d = p->head_dim;
  pd->g_q = p->h_q / p->h_kv;
  pd->dtype = p->dtype;
  pd->page_size = p->page_size; pd->max_pages = p->max_pages; pd->num_pages = p->num_pages;
  pd->cap = p->max_pages * p->page_size;
  pd->sm_scale = 1.f / std::sqrt((float)p->head_dim);
  return DASH_OK;
}

// A tensor that is written may not repeat itself.
bool repeats(long long stride, long long extent) { return stride == 0 && extent > 1; }
bool pool_repeats(const PagedDims& pd, const long long* s, int num_pages) {
  return repeats(s[0], num_pages) || repeats(s[1], pd.page_size) || repeats(s[2], pd.h_kv);
}

// Radians per position as a 64-bit fraction of a turn: x / 2 pi as an unevaluated sum of two doubles, each term's fraction in units of
// 2^-64.  (In 80-bit arithmetic the 64 pairs of a head cost 3.6 us a call.)  Of the magnitude, the sign behind it: hi - floor(hi) is
// exact for hi >= 0 only (1 - 1e-5 has no room for the last ten bits of 1e-5, and far positions multiply what is lost by 2^31).
constexpr double MAX_FREQ = 1099511627776.0;      // 2^40: what the sum of two leaves out stays below 2^-64 there
unsigned long long turn_fraction(double x) {
  constexpr double HI = 0.15915494309189535, LO = -9.839338337591243e-18;      // 1 / 2 pi
  constexpr double TWO64 = 18446744073709551616.0;
  const double m = std::fabs(x), hi = m * HI, lo = std::fma(m, HI, -hi) + m * LO;
  const unsigned long long f = (unsigned long long)((hi - std::floor(hi)) * TWO64) + (unsigned long long)(long long)(lo * TWO64);
  return x < 0 ? 0ull - f : f;
}

int make_rope(const dash_rope* r, int head_dim, RopeTable* rt) {
  if (!r || r->struct_size != sizeof(dash_rope)) return DASH_ERR_INVALID_ARG;
  if (r->pairs <= 0 || 2 * r->pairs > head_dim || r->axes < 1 || r->axes > ROPE_MAX_AXES) return DASH_ERR_INVALID_ARG;
  if ((r->interleaved != 0 && r->interleaved != 1) || !r->axis || !r->inv_freq) return DASH_ERR_INVALID_ARG;
  std::memset(rt, 0, sizeof(*rt));
  rt->pairs = r->pairs;
  rt->interleaved = r->interleaved;
  for (int i = 0; i < r->pairs; ++i) {
    if (r->axis[i] < 0 || r->axis[i] >= r->axes || !(std::fabs(r->inv_freq[i]) <= MAX_FREQ)) return DASH_ERR_INVALID_ARG;
    rt->axis[i] = (unsigned char)r->axis[i];
    rt->freq[i] = turn_fraction(r->inv_freq[i]);
  }
  return DASH_OK;
}

// A prefill shape as the rotation sees it: sizes, and the strides of the tensors that are given.  (Chunks, groups and the routing's
// limits on them are none of its business.)
int make_rope_dims(const dash_params* p, bool q, bool k, Dims* dm) {
  if (!p || p->struct_size != sizeof(dash_params)) return DASH_ERR_INVALID_ARG;
  if (p->batch <= 0 || p->batch > 65535 || p->seq_q <= 0 || p->seq_q != p->seq_kv || p->h_q <= 0 || p->h_kv <= 0) return DASH_ERR_INVALID_ARG;
  if (p->h_q % p->h_kv != 0) return DASH_ERR_INVALID_ARG;
  if (p->dtype != DASH_F32 && p->dtype != DASH_BF16) return DASH_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return DASH_ERR_UNSUPPORTED;
  if ((long long)p->batch * p->seq_q > 0x7fffffffLL) return DASH_ERR_UNSUPPORTED;      // (blocks of a grid)
  std::memset(dm, 0, sizeof(*dm));
  if ((q && !good_strides<3>(p->q_stride, p->dtype, dm->qs)) || (k && !good_strides<3>(p->k_stride, p->dtype, dm->ks)))
    return DASH_ERR_INVALID_ARG;
  dm->batch = p->batch; dm->seq_q = dm->seq_kv = p->seq_q;
  dm->h_q = p->h_q; dm->h_kv = p->h_kv; dm->d = p->head_dim;
  dm->dtype = p->dtype;
  return DASH_OK;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t workspace_bytes(const PagedDims& pd) {
  const size_t partials = pd.dtype == DASH_BF16 ? chunk_sm100_partial_bytes(pd) : chunk_generic_partial_bytes(pd);
  return align256(STATUS_REGION_BYTES) + align256(partials);
}

int check_paged_workspace(const PagedDims& pd, void* ws, size_t bytes) {
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) != 0 || bytes < workspace_bytes(pd)) return DASH_ERR_WORKSPACE;
  return DASH_OK;
}

}  // namespace

}  // namespace dash

using namespace dash;

extern "C" {

int dash_attn_rope(const dash_params* p, const dash_rope* rope, const int32_t* positions, const void* Q, const void* K,
                   void* Qout, void* Kout, int32_t inverse, void* stream) {
  Dims dm;
  int rc = make_rope_dims(p, Q != nullptr, K != nullptr, &dm);
  if (rc != DASH_OK) return rc;
  RopeTable rt;
  if ((rc = make_rope(rope, dm.d, &rt)) != DASH_OK) return rc;
  if (inverse != 0 && inverse != 1) return DASH_ERR_INVALID_ARG;
  if (!positions || !aligned4(positions) || (!Q && !K) || !Q != !Qout || !K != !Kout) return DASH_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(Qout) || !aligned16(Kout)) return DASH_ERR_INVALID_ARG;
  if ((Q && broadcasts(dm.qs, dm.batch, dm.seq_q, dm.h_q)) || (K && broadcasts(dm.ks, dm.batch, dm.seq_q, dm.h_kv)))
    return DASH_ERR_INVALID_ARG;
  if ((rc = validate_device()) != DASH_OK) return rc;
  StageRange nv("dash_attn: rotary positions");
  return cuda_status(launch_rope(dm, rt, positions, Q, K, Qout, Kout, inverse != 0, (cudaStream_t)stream));
}

int dash_attn_append_paged(const dash_paged_params* p, const dash_rope* rope, const int32_t* positions,
                           const int32_t* q_start, const int32_t* kv_len, const int32_t* page_table, const void* Q,
                           void* Qout, const void* K, const void* V, void* Kpool, void* Vpool, void* stream) {
  PagedDims pd;
  int rc = make_paged(p, &pd);
  if (rc != DASH_OK) return rc;
  RopeTable rt;
  std::memset(&rt, 0, sizeof(rt));
  if (rope && (rc = make_rope(rope, pd.d, &rt)) != DASH_OK) return rc;
  if (!q_start || !kv_len || !page_table || !Kpool || !Vpool) return DASH_ERR_INVALID_ARG;
  if (pd.rows > 0 && (!rope != !positions || !K || !V || !Q != !Qout)) return DASH_ERR_INVALID_ARG;
  if (!aligned4(positions) || !aligned4(q_start) || !aligned4(kv_len) || !aligned4(page_table)) return DASH_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(Qout) || !aligned16(K) || !aligned16(V) || !aligned16(Kpool) || !aligned16(Vpool))
    return DASH_ERR_INVALID_ARG;
  if (Q && (repeats(pd.os[0], pd.rows) || repeats(pd.os[1], pd.h_q))) return DASH_ERR_INVALID_ARG;
  if (Q == Qout && Q && (pd.os[0] != pd.qs[0] || pd.os[1] != pd.qs[1])) return DASH_ERR_INVALID_ARG;
  if (pool_repeats(pd, pd.ks, pd.num_pages) || pool_repeats(pd, pd.vs, pd.num_pages)) return DASH_ERR_INVALID_ARG;
  if ((rc = validate_device()) != DASH_OK) return rc;
  if (pd.rows == 0) return DASH_OK;
  StageRange nv("dash_attn: new tokens into pages");
  return cuda_status(launch_append(pd, rt, positions, q_start, kv_len, page_table, Q, Qout, K, V, Kpool, Vpool, (cudaStream_t)stream));
}

size_t dash_attn_paged_workspace_bytes(const dash_paged_params* p) {
  PagedDims pd;
  if (make_paged(p, &pd) != DASH_OK) return 0;
  return workspace_bytes(pd);
}

int dash_attn_attend_chunk_paged(const dash_paged_params* p, const void* Q, const void* Kpool, const void* Vpool,
                                 const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len, void* O, float* lse,
                                 void* workspace, size_t workspace_size, void* stream) {
  PagedDims pd;
  int rc = make_paged(p, &pd);
  if (rc != DASH_OK) return rc;
  if (!Kpool || !Vpool || !page_table || !q_start || !kv_len || (pd.rows > 0 && (!Q || !O))) return DASH_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(Kpool) || !aligned16(Vpool) || !aligned16(O)) return DASH_ERR_INVALID_ARG;
  if (!aligned4(page_table) || !aligned4(q_start) || !aligned4(kv_len) || !aligned4(lse)) return DASH_ERR_INVALID_ARG;
  if (repeats(pd.os[0], pd.rows) || repeats(pd.os[1], pd.h_q)) return DASH_ERR_INVALID_ARG;
  if ((rc = check_paged_workspace(pd, workspace, workspace_size)) != DASH_OK) return rc;
  if (pd.dtype == DASH_BF16 && !chunk_sm100_supported(pd)) return DASH_ERR_UNSUPPORTED;
  if ((rc = validate_device()) != DASH_OK) return rc;
  if (pd.rows == 0) return DASH_OK;
  StatusBlock* sb = reinterpret_cast<StatusBlock*>(workspace);
  float* partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + align256(STATUS_REGION_BYTES));
  StageRange nv("dash_attn: chunk attention over pages");
  if (pd.dtype == DASH_BF16)
    return cuda_status(launch_attend_chunk_sm100(pd, Q, Kpool, Vpool, page_table, q_start, kv_len, O, lse, partials, sb, (cudaStream_t)stream));
  return cuda_status(launch_attend_chunk_generic(pd, Q, Kpool, Vpool, page_table, q_start, kv_len, O, lse, partials, (cudaStream_t)stream));
}

int dash_attn_key_mass_paged(const dash_paged_params* p, const void* Q, const void* Kpool, const int32_t* page_table,
                             const int32_t* q_start, const int32_t* kv_len, const float* lse, float decay,
                             const float* mass_in, float* mass_out, void* workspace, size_t workspace_size, void* stream) {
  PagedDims pd;
  int rc = make_paged(p, &pd);
  if (rc != DASH_OK) return rc;
  if (!Kpool || !page_table || !q_start || !kv_len || !mass_out || !std::isfinite(decay)) return DASH_ERR_INVALID_ARG;
  if (pd.rows > 0 && (!Q || !lse)) return DASH_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(Kpool)) return DASH_ERR_INVALID_ARG;
  if (!aligned4(page_table) || !aligned4(q_start) || !aligned4(kv_len) || !aligned4(lse) || !aligned4(mass_in) || !aligned4(mass_out))
    return DASH_ERR_INVALID_ARG;
  if ((rc = check_paged_workspace(pd, workspace, workspace_size)) != DASH_OK) return rc;
  if (pd.dtype == DASH_BF16 && !chunk_sm100_supported(pd)) return DASH_ERR_UNSUPPORTED;
  if ((rc = validate_device()) != DASH_OK) return rc;
  StageRange nv("dash_attn: attention weight per cached token");
  if (pd.dtype == DASH_BF16)
    return cuda_status(launch_key_mass_sm100(pd, Q, Kpool, page_table, q_start, kv_len, lse, decay, mass_in, mass_out,
                                             reinterpret_cast<float*>(static_cast<char*>(workspace) + align256(STATUS_REGION_BYTES)),
                                             reinterpret_cast<StatusBlock*>(workspace), (cudaStream_t)stream));
  return cuda_status(launch_key_mass_generic(pd, Q, Kpool, page_table, q_start, kv_len, lse, decay, mass_in, mass_out, (cudaStream_t)stream));
}

int dash_attn_evict_paged(const dash_paged_params* p, int32_t keep, int32_t sinks, int32_t recent, const float* mass,
                          const int32_t* kv_len, const int32_t* page_table, const void* Kpool, const void* Vpool,
                          int32_t* kept, int32_t* new_len, const int32_t* dst_table, int32_t dst_max_pages,
                          int32_t dst_num_pages, void* Kdst, void* Vdst, float* mass_out, void* stream) {
  PagedDims pd;
  int rc = make_paged(p, &pd);
  if (rc != DASH_OK) return rc;
  if (keep <= 0 || sinks < 0 || recent < 0 || (long long)sinks + recent > keep) return DASH_ERR_INVALID_ARG;
  if (keep > (1 << 30)) return DASH_ERR_UNSUPPORTED;       // (a block's steps through `kept` stay within 32 bits)
  if (!mass || !kv_len || !page_table || !Kpool || !Vpool || !kept || !new_len || !dst_table || !Kdst || !Vdst) return DASH_ERR_INVALID_ARG;
  if (dst_max_pages <= 0 || dst_num_pages <= 0) return DASH_ERR_INVALID_ARG;
  const long long dst_cap = (long long)dst_max_pages * pd.page_size;
  if (dst_cap < (keep < pd.cap ? keep : pd.cap) || dst_cap > (1 << 25)) return DASH_ERR_INVALID_ARG;
  if (!aligned16(Kpool) || !aligned16(Vpool) || !aligned16(Kdst) || !aligned16(Vdst)) return DASH_ERR_INVALID_ARG;
  if (!aligned4(mass) || !aligned4(kv_len) || !aligned4(page_table) || !aligned4(kept) || !aligned4(new_len) || !aligned4(dst_table) ||
      !aligned4(mass_out))
    return DASH_ERR_INVALID_ARG;
  if ((long long)pd.batch * pd.h_kv * (((long long)(keep < pd.cap ? keep : pd.cap) + 63) / 64) > 0x7fffffffLL) return DASH_ERR_UNSUPPORTED;
  if (new_len == kv_len) return DASH_ERR_INVALID_ARG;
  EvictArgs a;
  a.in_place = dst_table == page_table;
  if (a.in_place && (Kdst != Kpool || Vdst != Vpool || dst_max_pages != pd.max_pages || dst_num_pages != pd.num_pages)) return DASH_ERR_INVALID_ARG;
  if (!a.in_place && mass_out == mass) return DASH_ERR_INVALID_ARG;
  if (pool_repeats(pd, pd.ks, dst_num_pages) || pool_repeats(pd, pd.vs, dst_num_pages)) return DASH_ERR_INVALID_ARG;
  if ((rc = validate_device()) != DASH_OK) return rc;
  a.keep = keep; a.sinks = sinks; a.recent = recent;
  a.mass = mass; a.kv_len = kv_len; a.page_table = page_table;
  a.pool[0] = (const char*)Kpool; a.pool[1] = (const char*)Vpool;
  a.kept = kept; a.new_len = new_len;
  a.dst_table = dst_table; a.dst_max_pages = dst_max_pages; a.dst_num_pages = dst_num_pages;
  a.dst[0] = (char*)Kdst; a.dst[1] = (char*)Vdst;
  a.mass_out = mass_out;
  StageRange nv("dash_attn: eviction");
  return cuda_status(launch_evict(pd, a, (cudaStream_t)stream));
}

}  // extern "C"
