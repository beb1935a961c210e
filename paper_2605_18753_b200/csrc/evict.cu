// Eviction from the paged cache by accumulated attention weight: per (sequence, KV head) the `keep` slots with the largest keys,
// then their K, V and mass rows moved to the front in order.
//
// Selection (evict_select_kernel): a mass becomes a 32-bit key whose unsigned order is the order of the floats (NaN lowest); slots
// kept in any case have the largest key of all, so one selection of `keep` slots with ties to the lower slot says everything.  The
// keep-th largest key is found digit by digit (four passes of eight bits, a histogram each).  A cluster of blocks serves a
// (sequence, KV head): every block holds its share of the keys in shared memory, so the mass is read from memory once; the
// blocks' histograms are summed over distributed shared memory.  Then every warp counts its stretch of the keys and, behind a scan
// over the cluster, writes its kept slots.  Bound by the latency of its passes where caches are short, by shared-memory atomics
// where they are long.
//
// Move (evict_move_kernel): bytes.  To other pages: blocks along the kept rows (4096 of each of 128 caches, 537 MB read and written: 94 us,
// 5.7 TB/s, 87 % of the measured copy).  In place: row j comes from slot kept[j] >= j, so one
// block that takes the rows in order, each batch in registers before any of it is written, never writes a row that it has yet
// to read; a (sequence, KV head) is divided among blocks by 64-byte columns of K and V instead, which nobody else touches.  16 x 8
// caches of 32768 slots to 4096, d 128, bf16: 191 us with the selection, 84 us of bytes (the rows of a batch wait for each other); of 4196 slots
// 172; caches that are not above the limit are written onto themselves (4096 slots: 158).
#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace dash {

namespace {

constexpr int SEL_THREADS = 512, SEL_WARPS = SEL_THREADS / 32;
constexpr int SEL_KEYS = 40960;              // keys of a block in shared memory (160 KiB); more are read again every pass
constexpr unsigned ALWAYS = 0xffffffffu;     // above the key of +inf (0xff800000)

__device__ __forceinline__ unsigned key_of(float x) {
  unsigned u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;              // NaN
  if (u == 0x80000000u) u = 0u;                                // -0 equals 0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

struct SelShared {
  unsigned hist[256 * 32];       // [bin][lane]: weights share their leading bits, so the lanes of a warp mostly meet in a few bins; a
                                 // count of its own per lane keeps them from waiting for one another
  unsigned bins[256];
  unsigned sum[2][256];          // this block's histogram, read by the whole cluster (two: a pass writes one while the other is read)
  unsigned scan[8];
  unsigned digit, left;
  unsigned counts[2];            // this block's keys above / at the threshold
  unsigned warp_n[2][SEL_WARPS];
};

__device__ __forceinline__ unsigned ld_cluster_u32(uint32_t addr) {
  unsigned v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

__global__ void __launch_bounds__(SEL_THREADS) evict_select_kernel(PagedDims pd, EvictArgs a, int cluster, int key_room) {
  extern __shared__ unsigned keys[];
  __shared__ SelShared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = (int)(blockIdx.x % cluster);
  const int grp = (int)(blockIdx.x / cluster), b = grp / pd.h_kv;
  chain_wait();
  const int n = min(max(__ldg(a.kv_len + b), 0), pd.cap);
  int* kept = a.kept + (long long)grp * a.keep;
  const int len = min(n, a.keep);
  for (int j = len + rank * SEL_THREADS + tid; j < a.keep; j += cluster * SEL_THREADS) kept[j] = -1;
  if (n <= a.keep) {             // (the same for all blocks of the cluster)
    for (int j = rank * SEL_THREADS + tid; j < n; j += cluster * SEL_THREADS) kept[j] = j;
    return;
  }
  const float* mass = a.mass + (long long)grp * pd.cap;
  const int lo = min(a.sinks, n), hi = max(n - a.recent, lo);
  // this block's share of the slots, and every warp's stretch of that
  const int share = (n + cluster - 1) / cluster, begin = min(rank * share, n), here = min(share, n - begin);
  const int stretch = (here + SEL_WARPS - 1) / SEL_WARPS, w0 = min(warp * stretch, here), w1 = min(w0 + stretch, here);
  const bool held = here <= key_room;
  auto key_at = [&](int k, float m) {
    const int slot = begin + k;
    return slot < lo || slot >= hi ? ALWAYS : key_of(m);
  };
  auto fresh = [&](int k) { return key_at(k, __ldg(mass + begin + k)); };
  auto key = [&](int k) { return held ? keys[k] : fresh(k); };

  unsigned prefix = 0, left = (unsigned)a.keep;      // digits found; how many of the keys that match them are still to be kept
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    for (int k = tid; k < 256 * 32; k += SEL_THREADS) sh.hist[k] = 0;
    __syncthreads();
    if (pass == 0) {
      for (int k0 = w0; k0 < w1; k0 += 256) {
        float m[8];                          // on their way at once (behind a condition of its own each would wait for the one before)
#pragma unroll
        for (int i = 0; i < 8; ++i) m[i] = __ldg(mass + begin + min(k0 + 32 * i + lane, w1 - 1));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int k = k0 + 32 * i + lane;
          if (k < w1) {
            const unsigned x = key_at(k, m[i]);
            if (held) keys[k] = x;
            atomicAdd(&sh.hist[(x >> 24) * 32 + lane], 1u);
          }
        }
      }
    } else {
#pragma unroll 8
      for (int k = w0 + lane; k < w1; k += 32) {
        const unsigned x = key(k);
        if ((x >> (shift + 8)) == prefix) atomicAdd(&sh.hist[((x >> shift) & 255u) * 32 + lane], 1u);
      }
    }
    __syncthreads();
    unsigned* sum = sh.sum[pass & 1];
    unsigned mine = 0;
    {
      // two threads a bin, sixteen lanes' counts each, every thread from another bank
      static_assert(SEL_THREADS == 512, "two threads per bin");
      const int bin = tid >> 1, half = tid & 1;
      unsigned n = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) n += sh.hist[bin * 32 + half * 16 + ((j + bin) & 15)];
      n += __shfl_xor_sync(0xffffffffu, n, 1);
      if (half == 0) sum[bin] = n;
      if (cluster == 1) {
        __syncthreads();
        if (tid < 256) mine = sum[tid];
      }
    }
    if (cluster > 1) {
      ptx::cluster_sync_all();
      if (tid < 256) {
        const uint32_t at = ptx::smem_u32(&sum[tid]);
        mine = 0;
        for (int c = 0; c < cluster; ++c) mine += ld_cluster_u32(ptx::map_to_rank(at, c));
      }
    }
    // keys whose digit is above this thread's: a suffix sum over the 256 bins (thread 0 takes the highest bin)
    if (tid < 256) sh.bins[tid] = mine;
    __syncthreads();
    unsigned v = 0, incl = 0;
    if (tid < 256) {
      v = sh.bins[255 - tid];
      incl = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
      }
      if (lane == 31) sh.scan[warp] = incl;
    }
    __syncthreads();
    if (tid < 256) {
      for (int w = 0; w < warp; ++w) incl += sh.scan[w];
      if (incl >= left && incl - v < left) {
        sh.digit = 255u - tid;
        sh.left = left - (incl - v);
      }
    }
    __syncthreads();
    prefix = (prefix << 8) | sh.digit;
    left = sh.left;
  }
  // keys above the threshold are kept, and the first `left` of those at it
  unsigned above = 0, at = 0;
#pragma unroll 8
  for (int k = w0 + lane; k < w1; k += 32) {
    const unsigned x = key(k);
    above += x > prefix;
    at += x == prefix;
  }
  above = __reduce_add_sync(0xffffffffu, above);
  at = __reduce_add_sync(0xffffffffu, at);
  if (lane == 0) {
    sh.warp_n[0][warp] = above;
    sh.warp_n[1][warp] = at;
  }
  __syncthreads();
  if (tid < 2) {
    unsigned s = 0;
    for (int w = 0; w < SEL_WARPS; ++w) s += sh.warp_n[tid][w];
    sh.counts[tid] = s;
  }
  unsigned above0 = 0, at0 = 0;        // ... before this warp's stretch
  if (cluster > 1) {
    ptx::cluster_sync_all();
    const uint32_t addr = ptx::smem_u32(&sh.counts[0]);
    for (int c = 0; c < rank; ++c) {
      const uint32_t far = ptx::map_to_rank(addr, c);
      above0 += ld_cluster_u32(far);
      at0 += ld_cluster_u32(far + 4);
    }
  }
  for (int w = 0; w < warp; ++w) {
    above0 += sh.warp_n[0][w];
    at0 += sh.warp_n[1][w];
  }
  const unsigned below = (1u << lane) - 1u;
#pragma unroll 4
  for (int k0 = w0; k0 < w1; k0 += 32) {
    const int k = k0 + lane;
    const unsigned x = k < w1 ? key(k) : 0u;
    const unsigned g = __ballot_sync(0xffffffffu, k < w1 && x > prefix), e = __ballot_sync(0xffffffffu, k < w1 && x == prefix);
    const unsigned ge = at0 + __popc(e & below);         // equals before this lane
    const bool take = (g >> lane & 1u) || ((e >> lane & 1u) && ge < left);
    if (take) kept[above0 + __popc(g & below) + min(ge, left)] = begin + k;
    above0 += __popc(g);
    at0 += __popc(e);
  }
  if (cluster > 1) ptx::cluster_sync_all();              // nobody leaves while its shared memory may be read
}

constexpr int MOVE_THREADS = 256, MOVE_ROWS = 64;

// A row of head_dim elements is `vecs` 16-byte vectors.  Slot `slot` of a sequence in pages `table`; nullptr where there is none.
__device__ __forceinline__ char* row_at(const char* pool, const int* table, int page_size, int num_pages, const long long* stride,
                                        int bytes, int slot, int r) {
  const int lp = slot / page_size, ph = __ldg(table + lp);
  if (ph < 0 || ph >= num_pages) return nullptr;
  return const_cast<char*>(pool) + ((long long)ph * stride[0] + (long long)(slot - lp * page_size) * stride[1] + r * stride[2]) * bytes;
}

// To other pages: a block moves MOVE_ROWS kept rows.  A thread takes two vectors of a row's K and the same two of its V, so that the row's
// addresses (two divisions, a list entry, two page-table entries) are worked out once for 64 bytes, and two rows at a time: the
// pools may be one, so the compiler would finish one copy before it starts the next.
__global__ void __launch_bounds__(MOVE_THREADS) evict_move_kernel(PagedDims pd, EvictArgs a, int per_group) {
  const int grp = blockIdx.x / per_group, part = blockIdx.x - grp * per_group, b = grp / pd.h_kv, r = grp - b * pd.h_kv;
  const int bytes = pd.dtype == DASH_BF16 ? 2 : 4, half = pd.d * bytes / 32, log_half = 31 - __clz(half);      // vectors of half a row
  chain_wait();
  const int len = min(min(max(__ldg(a.kv_len + b), 0), pd.cap), a.keep);
  if (part == 0 && r == 0 && threadIdx.x == 0) a.new_len[b] = len;
  const int j0 = part * MOVE_ROWS, j1 = min(j0 + MOVE_ROWS, len);
  const int* kept = a.kept + (long long)grp * a.keep;
  const int* from = a.page_table + (long long)b * pd.max_pages;
  const int* to = a.dst_table + (long long)b * a.dst_max_pages;
  const int v = (threadIdx.x & (half - 1)) * 16, step = MOVE_THREADS >> log_half;
  for (int j = j0 + (threadIdx.x >> log_half); j < j1; j += 2 * step) {
    uint4 x[2][4];
    char* d[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int jj = j + i * step;
      d[i][0] = d[i][1] = nullptr;
      if (jj >= j1) continue;
      const int src = kept[jj], sp = src / pd.page_size, st = src - sp * pd.page_size, dp = jj / pd.page_size, dt = jj - dp * pd.page_size;
      const int ph = __ldg(from + sp), dh = __ldg(to + dp);
      const bool there = ph >= 0 && ph < pd.num_pages;
      if (dh >= 0 && dh < a.dst_num_pages) {
        d[i][0] = a.dst[0] + (dh * pd.ks[0] + dt * pd.ks[1] + r * pd.ks[2]) * bytes + v;
        d[i][1] = a.dst[1] + (dh * pd.vs[0] + dt * pd.vs[1] + r * pd.vs[2]) * bytes + v;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) x[i][k] = make_uint4(0u, 0u, 0u, 0u);
      if (there) {
        const char* ks = a.pool[0] + (ph * pd.ks[0] + st * pd.ks[1] + r * pd.ks[2]) * bytes + v;
        const char* vs = a.pool[1] + (ph * pd.vs[0] + st * pd.vs[1] + r * pd.vs[2]) * bytes + v;
        x[i][0] = *reinterpret_cast<const uint4*>(ks);
        x[i][1] = *reinterpret_cast<const uint4*>(ks + half * 16);
        x[i][2] = *reinterpret_cast<const uint4*>(vs);
        x[i][3] = *reinterpret_cast<const uint4*>(vs + half * 16);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (d[i][0]) {
        *reinterpret_cast<uint4*>(d[i][0]) = x[i][0];
        *reinterpret_cast<uint4*>(d[i][0] + half * 16) = x[i][1];
        *reinterpret_cast<uint4*>(d[i][1]) = x[i][2];
        *reinterpret_cast<uint4*>(d[i][1] + half * 16) = x[i][3];
      }
  }
  if (a.mass_out)
    for (int j = j0 + threadIdx.x; j < j1; j += MOVE_THREADS)
      a.mass_out[(long long)grp * a.dst_max_pages * pd.page_size + j] = __ldg(a.mass + (long long)grp * pd.cap + kept[j]);
}

// In place: block (part, group); parts 0 .. 2 * columns - 1 are 64-byte columns of K and V, the last is the mass.
constexpr int COLUMN = 4;                    // vectors
constexpr int PLACE_THREADS = 512, PLACE_ROWS = PLACE_THREADS / COLUMN;

__global__ void __launch_bounds__(PLACE_THREADS) evict_place_kernel(PagedDims pd, EvictArgs a, int columns) {
  const int tid = threadIdx.x, parts = 2 * columns + 1, grp = blockIdx.x / parts, part = blockIdx.x - grp * parts;
  const int b = grp / pd.h_kv, r = grp - b * pd.h_kv;
  const int bytes = pd.dtype == DASH_BF16 ? 2 : 4;
  chain_wait();
  const int len = min(min(max(__ldg(a.kv_len + b), 0), pd.cap), a.keep);
  if (part == 0 && r == 0 && tid == 0) a.new_len[b] = len;
  const int* kept = a.kept + (long long)grp * a.keep;
  if (part == 2 * columns) {
    if (!a.mass_out) return;
    const float* src = a.mass + (long long)grp * pd.cap;
    float* dst = a.mass_out + (long long)grp * pd.cap;
    for (int j0 = 0; j0 < len; j0 += PLACE_THREADS) {
      const int j = j0 + tid;
      const float x = j < len ? src[kept[j]] : 0.f;
      __syncthreads();
      if (j < len) dst[j] = x;
      __syncthreads();
    }
    return;
  }
  const int kv = part / columns, v = (part - kv * columns) * COLUMN + tid % COLUMN;
  const long long* st = kv ? pd.vs : pd.ks;
  const char* pool = kv ? a.pool[1] : a.pool[0];
  const int* table = a.page_table + (long long)b * pd.max_pages;
  // two batches in registers: the next one is on its way while this one is written (its sources lie at or behind its own first
  // row, so behind everything that this batch writes)
  auto load = [&](int j, bool* there) {
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    *there = j < len;
    if (*there) {
      const char* s = row_at(pool, table, pd.page_size, pd.num_pages, st, bytes, kept[j], r);
      if (s) x = *reinterpret_cast<const uint4*>(s + v * 16);
    }
    return x;
  };
  bool there, there_next;
  uint4 x = load(tid / COLUMN, &there);
  for (int j0 = 0; j0 < len; j0 += PLACE_ROWS) {
    const int j = j0 + tid / COLUMN;
    const uint4 next = load(j + PLACE_ROWS, &there_next);
    __syncthreads();                         // the whole batch has been read
    if (there) {
      char* d = row_at(pool, table, pd.page_size, pd.num_pages, st, bytes, j, r);
      if (d) *reinterpret_cast<uint4*>(d + v * 16) = x;
    }
    x = next;
    there = there_next;
  }
}

}  // namespace

cudaError_t launch_evict(const PagedDims& pd, const EvictArgs& a, cudaStream_t st) {
  // Blocks per (sequence, KV head): enough to hold the keys on chip, and then as many (up to the portable cluster of eight, 4096 slots
  // each) as are resident at once, two per SM: a pass costs its barriers and scans whatever it counts.  16 x 8 caches of up to 32768
  // slots: eight blocks each 65 us, two 47 (35 with the loads in flight together).
  const int groups = pd.batch * pd.h_kv;
  int cluster = 1;
  while (cluster < 8 && (pd.cap > SEL_KEYS * cluster || (pd.cap > 4096 * cluster && groups * cluster * 2 <= 2 * current_sm_count()))) cluster *= 2;
  const int share = (pd.cap + cluster - 1) / cluster;
  const int room = share < SEL_KEYS ? share : SEL_KEYS;
  static std::atomic<unsigned long long> configured{0};
  if (cudaError_t e = allow_dynamic_smem(evict_select_kernel, SEL_KEYS * sizeof(unsigned), configured); e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(groups * cluster));
  cfg.blockDim = dim3(SEL_THREADS);
  cfg.dynamicSmemBytes = (size_t)room * sizeof(unsigned);
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  cudaError_t e = cudaLaunchKernelEx(&cfg, evict_select_kernel, pd, a, cluster, room);
  count_launch();
  if (e != cudaSuccess) return e;
  if (a.in_place) {
    const int columns = pd.d * (pd.dtype == DASH_BF16 ? 2 : 4) / 16 / COLUMN;
    e = launch_chained(evict_place_kernel, dim3((unsigned)(groups * (2 * columns + 1))), dim3(PLACE_THREADS), 0, st, pd, a, columns);
  } else {
    const int rows = MOVE_ROWS, per_group = ((a.keep < pd.cap ? a.keep : pd.cap) + rows - 1) / rows;
    e = launch_chained(evict_move_kernel, dim3((unsigned)((long long)groups * per_group)), dim3(MOVE_THREADS), 0, st, pd, a, per_group);
  }
  count_launch();
  return e;
}

}  // namespace dash
