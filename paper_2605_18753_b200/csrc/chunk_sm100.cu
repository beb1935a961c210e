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
//   a unit of at most TQ tokens (decode): both stages hold the same rows and take every other K / V tile; their results are joined.
//
// Schedule: the K / V tiles of all units, one behind another, are cut into equal ranges, one per block (a persistent grid of one
// block per SM).  Sequences of any mix of lengths, one long cache or many short ones, keep every SM busy to the end.  What a block
// has of a unit that is cut is a partial result (m, l, O); a second kernel joins those of each cut unit in the order of the cuts.
// Only the two ends of a range can be cut, so partial results take two places per block, whatever the problem.  (Joined by the last
// block to arrive instead, inside this kernel: 8 to 14 us of fences, counters and dependent loads at the end of every block.)
//
// Warp roles (384 threads): warps 0-3 and 4-7 softmax of stage 0 / 1, a row per thread; warp 8 loads Q and K, warp 9 V (TMA, a box
// per page or per 128 tokens of one), warps 10 and 11 issue the MMAs of stage 0 / 1 (one warp for both: a wait for one stage's
// weights held up the other's scores).  P is written over S in tensor memory (bf16) and is the A operand of P V; its first three
// quarters go to the product while the last is formed.
//
// What bounds it: 4096 rows over 16384 slots, 32/8 heads, d 128 (962 GFLOP): 0.88 to 0.90 ms in a long loop, 1.08 PFLOP/s, 78 % of the
// measured sustained cuBLAS rate (the power limit; the first calls of a cool GPU take 765 us, 75 % of the burst).  Of those 765, the
// same schedule without the softmax arithmetic takes 608 us, without all but one MMA of each product 665, so the softmax threads' chain of a step (scores out of tensor memory, maximum, 128
// exponentials, weights back) is the longer of the two.  Tried and slower: steps of 64 slots with two score buffers (the scores'
// products then read Q from shared memory twice as often), two warpgroups per stage (1.18 ms: 96 registers a thread), the weights
// formed ahead of the maximum.  One token of each of 16 caches of up to 65536 slots (2.4 GB): 371 to 421 us
// by GPU, 5.7 to 6.5 TB/s, 87 to 99 % of the measured copy.
// Rounding: the weights meet V as one bf16 term (2^-8 of each at most, against their unrounded sum), because a second term would be half of
// the products again.  O against float64 (2-norm): 2.3e-3, of which its own rounding to bf16 is 1.7e-3.
// Every wait is bounded; one that runs out raises DASH_ERR_TIMEOUT in the status word, and every role leaves.
#include <cuda.h>

#include "paged.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"

namespace dash {

namespace {

constexpr int NT = 128;                      // slots per K / V tile
constexpr int KST = 2, VST = 2;              // ring depths
constexpr int P_AHEAD = 96;                  // slots of P whose product with V starts before the rest is there
constexpr int THREADS = 384;
constexpr int REGS_SOFTMAX = 208, REGS_SERVICE = 88;
static_assert(256 * REGS_SOFTMAX + 128 * REGS_SERVICE <= THREADS * 168, "what the block was launched with");
constexpr uint32_t TMEM_COLS = 512;          // S0 [0,128), S1 [128,256), O0 [256,256+d), O1 behind it
constexpr int OFF_ROW = 0x3fffffff;          // slots that a row sees which is not there: more than any cache has
constexpr float RESCALE_LOG2 = 8.f;          // the running maximum moves only when it grew by more than this
constexpr int MAX_SLOTS = 4096;              // unit slots (see the plan) of one launch
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Which of the 16 pairs of a tensor-memory load take their exponentials on the FMA pipe (exp2_fma): every fourth.  4096 rows over 16384
// slots, 32/8 heads, d 128: none 784 us, one in eight 777, in four 761, three in eight 810.
__host__ __device__ constexpr bool on_fma(int pair) { return pair % 4 == 3; }

enum Bar { Q_FULL = 0, Q_EMPTY, K_FULL, K_EMPTY = K_FULL + KST, V_FULL = K_EMPTY + KST, V_EMPTY = V_FULL + VST, S_FULL = V_EMPTY + VST,
           P_FULL = S_FULL + 2, PV_DONE = P_FULL + 4, O_FREE = PV_DONE + 2, MEET = O_FREE + 2, E_DONE, DRAIN = E_DONE + 8, V_SEEN = DRAIN + 2,
           N_BARS };      // P: [stage][part]; E: [stage][warp]

struct Misc {
  unsigned long long bar[N_BARS];
  uint32_t tmem_base;
  int abort_flag;
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
  struct Cut* cuts;
  StatusBlock* sb;
  long long hold;                  // test hook: clocks that V tiles of one parity are held back (0: none)
  int hold_odd;
  int inject;                      // test hook: the fourth K tile of a block is never loaded (the waits for it run out)
  long long wait_limit;            // clocks that a bounded wait may spin
};

// One block's share of a unit.
struct Piece {
  int b, r, t;                     // sequence, KV head, unit of the sequence
  int k0, len, n;                  // first K / V tile and number of them; the unit's
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

// The pieces of a block's range, in order: a position, from which piece() says the rest (little of it is live inside the loops).
struct Walk {
  int left, k0, slot, r;           // tiles left of the range; first tile of the piece, its unit's slot and KV head
  __device__ __forceinline__ Walk(const ChunkArgs& a, const Plan& pl) {
    left = (int)(pl.end - pl.begin);
    k0 = slot = r = 0;
    if (left <= 0) return;
    r = (int)(pl.begin / pl.total);
    const int rest = (int)(pl.begin - (long long)r * pl.total);
    int lo = 0, hi = a.n_slots;                // last slot with pref <= rest that has tiles
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (pl.pref[mid] <= rest) lo = mid; else hi = mid;
    }
    slot = lo;
    k0 = rest - pl.pref[lo];
  }
  __device__ __forceinline__ Piece piece(const ChunkArgs& a, const Plan& pl) const {
    Piece p;
    p.r = r;
    p.b = pl.seq[slot];
    p.s = load_seq(a.pd, a.q_start, a.kv_len, p.b);
    const int TT = 2 * a.TQ;
    p.t = slot + a.slot0 - (p.s.q0 / TT + p.b);
    p.n = pl.pref[slot + 1] - pl.pref[slot];
    p.k0 = k0;
    p.len = min(p.n - k0, left);
    p.tokens = min(TT, p.s.q_len - p.t * TT);
    p.two = p.tokens > a.TQ;
    return p;
  }
  __device__ __forceinline__ bool done() const { return left <= 0; }
  __device__ __forceinline__ void next(const ChunkArgs& a, const Plan& pl) {
    left -= min(pl.pref[slot + 1] - pl.pref[slot] - k0, left);
    k0 = 0;
    if (left <= 0) return;
    do {
      if (++slot == a.n_slots) {
        slot = 0;
        ++r;
      }
    } while (pl.pref[slot + 1] == pl.pref[slot]);
  }
};

// Partial results of a block: place 0 a unit begun by an earlier block, 1 one that later blocks go on with, each for two stages;
// 2 and 3 in turn the second stage's share of whole units in turns.
constexpr int PARTS = 6;
template <int HD> __host__ __device__ constexpr long long partial_floats() { return 128LL * (HD + 2); }
template <int HD>
__device__ __forceinline__ float* partial_at(const ChunkArgs& a, int block, int place, int stage) {
  return a.partials + ((long long)block * PARTS + (place < 2 ? 2 * place + stage : place + 2)) * partial_floats<HD>();
}

// What the joining kernel needs to know of the unit that a block cuts at its end.
struct Cut {
  int blocks;                      // that hold a part of it (0: the block cuts no unit)
  int row0, tokens, r, two, pad[3];
};

__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + __log2f(l)) * LN2; }      // (NaN stays NaN)
__device__ __forceinline__ float reciprocal(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Maxima that pass a NaN on, as the sums do: a row with one among its scores is NaN, not a row without keys.
__device__ __forceinline__ float max2(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
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
  auto wait_all = [&](uint32_t barrier, uint32_t parity) { return ptx::mbar_wait_warp(barrier, parity, abort_flag, a.wait_limit); };
  const int g_q = pd.g_q, TQ = a.TQ, TT = 2 * TQ;

  if (tid == 0) {
    misc->abort_flag = (sbase & 1023u) != 0u;
    for (int i = 0; i < N_BARS; ++i) ptx::mbar_init(bar(i), i >= P_FULL && i < PV_DONE ? 4 : i >= O_FREE && i < MEET ? 4 : i == MEET ? 8 :
                                                        i == Q_EMPTY || (i >= K_EMPTY && i < V_FULL) || (i >= V_EMPTY && i < S_FULL) || i == V_SEEN ? 2 : 1);
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

  Walk walk(a, pl);

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
      for (; ok && !walk.done(); walk.next(a, pl)) {
        const Piece p = walk.piece(a, pl);
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
          if (is_k && a.inject && cnt == 3) {
            ok = false;
            break;
          }
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
          if (!is_k && a.hold > 0 && (cnt & 1) == a.hold_odd)
            for (const long long t0 = clock64(); clock64() - t0 < a.hold;) {}
          if (lane == 0) ptx::mbar_arrive_expect_tx(bar(full + st), LY::KV_TILE);
          __syncwarp();
          if (lane < boxes) {
            const uint32_t dst = ring + st * LY::KV_TILE + lane * a.box * 128;
#pragma unroll
            for (int h = 0; h < HD / 64; ++h)
              ptx::tma_load_4d(dst + h * (LY::KV_TILE / (HD / 64)), tm, bar(full + st), h * 64, p.r, tok, page);
          }
        }
      }
      // Where a wait has run out, here or in another warp, the copies already issued land (bounded) before the block retires.
      if (lane == 0) {
        for (int c = max(0, cnt - ST); c < cnt; ++c)
          for (int k = 0; k < 200000 && !ptx::mbar_try_wait(bar(full + c % ST), (c / ST) & 1); ++k) {}
        if (is_k && q_cnt > 0)
          for (int k = 0; k < 200000 && !ptx::mbar_try_wait(bar(Q_FULL), (q_cnt - 1) & 1); ++k) {}
      }
    } else {
      // =========================== MMA issuers: warp 10 stage 0, warp 11 stage 1 ===========================
      constexpr uint32_t IDESC_QK = ptx::idesc_bf16_f32(128, NT, false, false);
      constexpr uint32_t IDESC_PV = ptx::idesc_bf16_f32(128, HD, false, true);
      const int s = warp - 10;
      const uint64_t qd0 = ptx::smem_desc_sw128(sbase, 16, 1024);
      const uint64_t kd0 = ptx::smem_desc_sw128(sbase + LY::OFF_K, 16, 1024);
      const uint64_t vd0 = ptx::smem_desc_sw128(sbase + LY::OFF_V, NT * 128, 1024);
      const uint32_t s_tmem = tmem + s * 128, o_tmem = tmem + 256 + s * HD;
      const bool lead = ptx::elect_one();
      int base = 0, q_cnt = 0, it = 0;        // K / V tiles of earlier pieces; pieces; steps so far
      bool ok = true;
      for (; ok && !walk.done(); walk.next(a, pl)) {
        const Piece p = walk.piece(a, pl);
        const int steps = p.two ? p.len : s == 0 ? (p.len + 1) / 2 : p.len / 2;
        const uint64_t qd = qd0 + (uint64_t)((p.two && s ? LY::Q_TILE : 0u) >> 4);
        auto tile_of = [&](int i) { return base + (p.two ? i : 2 * i + s); };
        // A tile's place in its ring is free once both stages have said so; in turns one stage says it for both.
        auto release = [&](int b) {
          ptx::mma_commit(bar(b));
          if (!p.two) ptx::mma_commit(bar(b));
        };
        auto k_here = [&](int i) {
          const int c = tile_of(i);
          return wait_all(bar(K_FULL + c % KST), (c / KST) & 1);
        };
        auto qk = [&](int i) {
          const int st = tile_of(i) % KST;
          if (lead) {
            const uint64_t kd = kd0 + (uint64_t)((st * LY::KV_TILE) >> 4);
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {
              const uint64_t off = (uint64_t)(((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4);
              ptx::mma_bf16_ss(s_tmem, qd + off, kd + off, IDESC_QK, k > 0 ? 1u : 0u);
            }
            ptx::mma_commit(bar(S_FULL + s));
            release(K_EMPTY + st);
            if (i + 1 == steps) ptx::mma_commit(bar(Q_EMPTY));           // the piece's last product with its queries
          }
          __syncwarp();
        };
        // In turns a stage waits for its own V tiles only, and behind an odd number of them the places of the ring change owner: the tile
        // before in a place was then the other stage's.  While that one is still on its way, the phase that this stage would wait for
        // looks like the one two before it, and the wait would pass at once.  So the stages tell each other when the last V tile of a
        // piece is here, and nobody starts the next piece (its scores, from which the clearing of a tail follows, included) before.
        // (K needs no such word: the queries that come first are loaded when all products with the ones before, and so with all K
        // tiles before, are over.)
        ok = wait_all(bar(Q_FULL), q_cnt & 1) && (q_cnt == 0 || wait_all(bar(V_SEEN), (q_cnt - 1) & 1)) && (steps == 0 || k_here(0));
        if (!ok) break;
        ptx::tc_fence_after();
        if (steps > 0) qk(0);
        else if (lead) {
          ptx::mbar_arrive(bar(Q_EMPTY));
          ptx::mbar_arrive(bar(V_SEEN));
        }
        for (int i = 0; i < steps; ++i) {
          // Everything but P is waited for ahead, so that nothing stands between the last half of P and the next scores.
          const int c = tile_of(i), st = c % VST;
          ok = wait_all(bar(V_FULL + st), (c / VST) & 1);
          if (ok && i + 1 == steps && lead) ptx::mbar_arrive(bar(V_SEEN));
          ok = ok && (i + 1 == steps || k_here(i + 1));
          // the first product of a unit overwrites O: its epilogue must have read the last one's
          if (ok && i == 0 && q_cnt > 0) ok = wait_all(bar(O_FREE + s), (q_cnt - 1) & 1);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            if (!(ok = ok && wait_all(bar(P_FULL + 2 * s + half), (it + i) & 1))) break;
            ptx::tc_fence_after();
            if (lead) {
              const uint64_t vd = vd0 + (uint64_t)((st * LY::KV_TILE) >> 4);
#pragma unroll
              for (int k = 0; k < NT / 16; ++k)
                if ((k >= P_AHEAD / 16) == (half == 1))
                  ptx::mma_bf16_ts(o_tmem, s_tmem + k * 8, vd + (uint64_t)((k * 16 * 128) >> 4), IDESC_PV, (i > 0 || k > 0) ? 1u : 0u);
              if (half) {
                ptx::mma_commit(bar(PV_DONE + s));
                release(V_EMPTY + st);
              }
            }
            __syncwarp();
          }
          if (!ok) break;
          if (i + 1 < steps) qk(i + 1);
        }
        __syncwarp();
        base += p.len;
        it += steps;
        ++q_cnt;
      }
      // what has been issued is let run out (bounded) before tensor memory goes back, whoever gave up
      if (lead) ptx::mma_commit(bar(DRAIN + s));
      for (int k = 0; k < 200000 && !ptx::mbar_try_wait(bar(DRAIN + s), 0); ++k) {}
      __syncwarp();
    }
  } else {
    // =========================== softmax, epilogue ===========================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFTMAX));
    const int s = warp >> 2, m = tid & 127;            // stage; row of the tile = TMEM lane
    const int mt = m / g_q, hh = m - mt * g_q;         // token of the row tile, head of the group
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_addr = lane_addr + s * 128, o_addr = lane_addr + 256 + s * HD;
    const float c1 = pd.sm_scale * LOG2E;
    // One arrival per warp: those of 32 lanes are taken one after another.
    auto arrive = [&](int b) {
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(b));
    };
    int base = 0, it = 0, meets = 0, turns = 0;
    if (tid == 0) a.cuts[blk].blocks = 0;
    bool ok = true;
    for (; ok && !walk.done(); walk.next(a, pl)) {
      float m_used = -INFINITY, l = 0.f;
      int steps, len;
      bool two, warp_on;
      {
      const Piece p = walk.piece(a, pl);
      two = p.two;
      len = p.len;
      steps = two ? len : s == 0 ? (len + 1) / 2 : len / 2;
      const int first = two && s ? TQ : 0;             // first token of this stage's rows in the unit
      const bool row_on = mt < TQ && first + mt < p.tokens;
      warp_on = __any_sync(0xffffffffu, row_on);
      // Slots that the row sees, from the piece's first tile of this stage on (rows that are not there never ask for a mask), the
      // fewest of the warp, and the slots that hold anything.
      const int kv0 = (p.k0 + (two ? 0 : s)) * NT, stride = two ? NT : 2 * NT;
      int seen = (!row_on ? OFF_ROW : (int)min(max((long long)p.s.kv - p.s.q_len + p.t * TT + first + mt + 1, 0LL), (long long)p.s.valid)) - kv0;
      int fewest = __reduce_min_sync(0xffffffffu, seen), held = p.s.valid - kv0, c = base + (two ? 0 : s);
      // The two warps of a scheduler share its exponential unit.  Left alone they fall into step, both at their exponentials, then both
      // waiting for products: so they take turns.
      auto my_turn = [&]() {
        if (two && (s == 1 || turns > 0)) wait_all(bar(E_DONE + 4 * (1 - s) + (warp & 3)), (s == 1 ? turns : turns - 1) & 1);
      };
      auto turn_over = [&]() {
        if (two) {
          arrive(E_DONE + 4 * s + (warp & 3));
          ++turns;
        }
      };
      for (int i = 0; i < steps; ++i, seen -= stride, fewest -= stride, held -= stride, c += two ? 1 : 2) {
        ok = wait_all(bar(S_FULL + s), (it + i) & 1);      // (the stage's product with V of the step before is done as well)
        if (!ok) break;
        // Stale rows behind the cache's end must not meet P = 0 as NaN: they are cleared in the tile.  (Not before the wait above: the
        // tile before in this place of the ring may not even have arrived, and the phase bit could not tell its load from this one's.  Behind it
        // that tile is here: it was this stage's of the step before, or one of a piece before, see V_SEEN.)
        if (held < NT) {
          ok = wait_all(bar(V_FULL + c % VST), (c / VST) & 1);
          if (!ok) break;
          if (m >= held) {
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
          uint32_t sr[NT];
#pragma unroll
          for (int q = 0; q < NT / 32; ++q) {
            uint32_t* part = sr + 32 * q;
            DASH_TMEM_LD32(part, s_addr + 32 * q);
          }
          ptx::tmem_wait_ld();
          if (fewest < NT) {
#pragma unroll
            for (int k = 0; k < NT; ++k)
              if (k >= seen) sr[k] = 0xff800000u;       // -inf
          }
          float ch[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) ch[k] = __uint_as_float(sr[k]);
#pragma unroll
          for (int q = 8; q + 16 <= NT; q += 16)
#pragma unroll
            for (int k = 0; k < 8; ++k) ch[k] = max3(ch[k], __uint_as_float(sr[q + k]), __uint_as_float(sr[q + k + 8]));
#pragma unroll
          for (int k = 0; k < 8; ++k) ch[k] = max2(ch[k], __uint_as_float(sr[NT - 8 + k]));
          const float top = max3(max3(ch[0], ch[1], ch[2]), max3(ch[3], ch[4], ch[5]), max2(ch[6], ch[7])) * c1;
          float corr = 1.f;
          bool moved = false;
          // (a NaN among the scores moves it too, and stays; rows that are not there, whose `seen` is beyond any cache, never do)
          if (!(top <= m_used + RESCALE_LOG2) && seen < OFF_ROW / 2) {
            const float now = max2(m_used, top);
            corr = exp2f(m_used - now);                // 0 when nothing was accumulated yet
            m_used = now;
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
          my_turn();
          const float off = m_used == -INFINITY ? 0.f : -m_used;
          const float2 c1v = make_float2(c1, c1), offv = make_float2(off, off);
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int q = 0; q < NT / 32; ++q) {
            uint32_t pk[16];
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              const float2 x = __ffma2_rn(make_float2(__uint_as_float(sr[32 * q + k]), __uint_as_float(sr[32 * q + k + 1])), c1v, offv);
              const float2 e = on_fma(k >> 1) ? exp2_fma(x) : make_float2(exp2f(x.x), exp2f(x.y));
              sum[(k >> 1) & 1] = __fadd2_rn(sum[(k >> 1) & 1], e);
              const __nv_bfloat162 hv = __floats2bfloat162_rn(e.x, e.y);
              pk[k >> 1] = *reinterpret_cast<const uint32_t*>(&hv);
            }
            ptx::tmem_st_n<16>(s_addr + 16 * q, pk);
            if (q == P_AHEAD / 32 - 1) {               // the first part goes ahead
              ptx::tmem_wait_st();
              ptx::tc_fence_before();
              arrive(P_FULL + 2 * s);
            }
          }
          turn_over();
          const float2 ls = __fadd2_rn(sum[0], sum[1]);
          l += ls.x + ls.y;
          ptx::tmem_wait_st();
          ptx::tc_fence_before();
        }
        if (!warp_on) {
          my_turn();
          turn_over();
          arrive(P_FULL + 2 * s);
        }
        arrive(P_FULL + 2 * s + 1);
      }
      }
      if (!ok) break;
      // ---- the unit's rows, or what this block has of them
      const Piece p = walk.piece(a, pl);
      const int first = p.two && s ? TQ : 0, i_row = p.t * TT + first + mt;
      const bool row_on = mt < TQ && first + mt < p.tokens;
      if (steps > 0) {
        ok = wait_all(bar(PV_DONE + s), (it + steps - 1) & 1);
        if (!ok) break;
        ptx::tc_fence_after();
      }
      const bool whole = p.len == p.n;
      const long long row = (long long)p.s.q0 + i_row, head = (long long)p.r * g_q + hh;
      // Output rows of this thread's group of four lanes (offset in O; -1: not a row).  A store of every lane's own row touches 32 lines
      // an instruction; four lanes first exchange their 16-byte pieces, then write 64 bytes of each other's rows.
      long long oofs[4];
      {
        const long long mine = row_on ? row * pd.os[0] + head * pd.os[1] : -1;
#pragma unroll
        for (int k = 0; k < 4; ++k) oofs[k] = __shfl_sync(0xffffffffu, mine, (lane & ~3) + k);
      }
      auto store64 = [&](int col, uint32_t (&w)[16]) {         // 32 columns from `col` on, packed; the whole warp
#pragma unroll
        for (int step = 1; step < 4; step <<= 1) {
          const bool up = lane & step;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (k & step) continue;
#pragma unroll
            for (int q = 0; q < 4; ++q) {                      // piece k of the upper lane against piece k + step of the lower one
              const uint32_t give = up ? w[k * 4 + q] : w[(k + step) * 4 + q];
              const uint32_t got = __shfl_xor_sync(0xffffffffu, give, step);
              if (up) w[k * 4 + q] = got; else w[(k + step) * 4 + q] = got;
            }
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (oofs[k] >= 0)
            *reinterpret_cast<uint4*>(a.O + oofs[k] + col + (lane & 3) * 8) = make_uint4(w[k * 4], w[k * 4 + 1], w[k * 4 + 2], w[k * 4 + 3]);
        __syncwarp();
      };
      if (whole && p.two) {
        const float inv = reciprocal(l);
#pragma unroll 1
        for (int q = 0; q < HD / 32 && warp_on; ++q) {
          uint32_t o[32], w[16];
          DASH_TMEM_LD32(o, o_addr + q * 32);
          ptx::tmem_wait_ld();
#pragma unroll
          for (int k = 0; k < 16; ++k) w[k] = pack2(__uint_as_float(o[2 * k]) * inv, __uint_as_float(o[2 * k + 1]) * inv);
          store64(q * 32, w);
        }
        if (row_on && a.lse) a.lse[row * pd.h_q + head] = lse_of(m_used, l);
        ptx::tc_fence_before();
        arrive(O_FREE + s);
      } else {
        // partial result: O unnormalised, four columns of all rows one behind another, then (m, l)
        auto keep_part = [&](float* part) {
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
                  __stcg(reinterpret_cast<float4*>(part) + ((q * 32 + k) >> 2) * 128 + m,
                         make_float4(__uint_as_float(o[k]), __uint_as_float(o[k + 1]), __uint_as_float(o[k + 2]), __uint_as_float(o[k + 3])));
              }
            }
            if (row_on) __stcg(reinterpret_cast<float2*>(part + 128 * HD) + m, make_float2(m_used, l));
          }
        };
        if (!whole) {
          keep_part(partial_at<HD>(a, blk, p.k0 > 0 ? 0 : 1, s));
          if (tid == 0 && p.k0 == 0) {
            const long long end = (long long)p.r * pl.total + pl.pref[walk.slot] + p.n;
            Cut c;
            c.blocks = (int)((end * G - 1) / pl.all) - blk + 1;      // up to the one whose range holds the unit's last tile
            c.row0 = p.s.q0 + p.t * TT;
            c.tokens = p.tokens;
            c.r = p.r;
            c.two = p.two;
            a.cuts[blk] = c;
          }
        } else {
          // a whole unit in turns: the first stage joins what the second has left
          float* part = partial_at<HD>(a, blk, 2 + (meets & 1), 0);
          if (s == 1) keep_part(part);
          __threadfence_block();
          arrive(MEET);
          if (!(ok = wait_all(bar(MEET), meets++ & 1))) break;       // (so nobody is more than one such unit ahead: two places do)
          if (s == 0 && warp_on) {
            float2 other = make_float2(-INFINITY, 0.f);
            if (row_on) other = __ldcg(reinterpret_cast<const float2*>(part + 128 * HD) + m);
            const float top = max2(m_used, other.x);
            const float w0 = m_used == -INFINITY ? 0.f : exp2f(m_used - top), w1 = other.x == -INFINITY ? 0.f : exp2f(other.x - top);
            const float sm = fmaf(l, w0, other.y * w1), inv = reciprocal(sm);
#pragma unroll 1
            for (int q = 0; q < HD / 32; ++q) {
              uint32_t o[32], w[16];
              float4 x[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (other.x != -INFINITY) x[k] = __ldcg(reinterpret_cast<const float4*>(part) + (q * 8 + k) * 128 + m);
              }
              __syncwarp();
              DASH_TMEM_LD32(o, o_addr + q * 32);
              ptx::tmem_wait_ld();
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const float f0 = w0 * inv, f1 = w1 * inv;
                w[2 * k] = pack2(fmaf(x[k].x, f1, __uint_as_float(o[4 * k]) * f0), fmaf(x[k].y, f1, __uint_as_float(o[4 * k + 1]) * f0));
                w[2 * k + 1] = pack2(fmaf(x[k].z, f1, __uint_as_float(o[4 * k + 2]) * f0), fmaf(x[k].w, f1, __uint_as_float(o[4 * k + 3]) * f0));
              }
              store64(q * 32, w);
            }
            if (row_on && a.lse) a.lse[row * pd.h_q + head] = lse_of(top, sm);
          }
        }
        ptx::tc_fence_before();
        arrive(O_FREE + s);
      }
      base += p.len;
      it += steps;
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

// Joins the partial results of a cut unit: block (x, y) the unit that attention block x cuts at its end, its y-th share.
//   a unit of two row tiles: 32 columns of all rows, a row per thread, part after part (few where there are many such units; where one is
//   all there is, the parts are a chain: 32 and 33 tokens over 65536 slots, 4 heads on one KV head, 78 and 193 us in all, with 8 KV
//   heads 84 and 104);
//   fewer rows (in up to 2 x 148 parts, where one long cache is all there is): a share of the rows, a thread four columns of one,
//   neighbouring threads neighbouring rows (as the parts lie), and what is left of the threads as P groups that take every P-th part and
//   meet in shared memory, so that a hundred parts are no chain of a hundred loads (16 tokens over 27,000 slots: 34 us in all, 73
//   with this case done as the other; shares by 32, or blocks of 512 threads, 28 to 31, but up to 4 us more where the parts are few).
constexpr int JOIN_THREADS = 256, JOIN_SHARES = 16;
template <int HD>
__global__ void __launch_bounds__(JOIN_THREADS) chunk_join_kernel(const __grid_constant__ ChunkArgs a) {
  constexpr int C4 = HD / 4;                          // pieces of four columns
  __shared__ float4 out[JOIN_THREADS];                // [P][row][piece]
  __shared__ float2 stat[JOIN_THREADS];               // [P][row]
  static_assert(128 / JOIN_SHARES * C4 <= JOIN_THREADS, "a share is no more than a piece per thread");
  const PagedDims& pd = a.pd;
  chain_wait();
  const int first = blockIdx.x, tid = threadIdx.x;
  const Cut c = a.cuts[first];
  if (c.blocks == 0) return;
  if (c.two) {
    const int col = blockIdx.y * 32, stage = tid >> 7, m = tid & 127, token = stage * a.TQ + m / pd.g_q;
    if (col >= HD || m >= a.TQ * pd.g_q || token >= c.tokens) return;
    float mx = -INFINITY, sm = 0.f;
    float4 acc[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int k = 0; k < c.blocks; ++k) {
      const float* part = partial_at<HD>(a, first + k, k == 0 ? 1 : 0, stage);
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(part + 128 * HD) + m);
      float4 x[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = __ldcg(reinterpret_cast<const float4*>(part) + (col / 4 + q) * 128 + m);
      if (ml.x != -INFINITY) {               // (a part without a key has nothing in its place)
        const float top = max2(mx, ml.x), corr = exp2f(mx - top), w = exp2f(ml.x - top);
        mx = top;
        sm = fmaf(ml.y, w, sm * corr);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          acc[q].x = fmaf(x[q].x, w, acc[q].x * corr); acc[q].y = fmaf(x[q].y, w, acc[q].y * corr);
          acc[q].z = fmaf(x[q].z, w, acc[q].z * corr); acc[q].w = fmaf(x[q].w, w, acc[q].w * corr);
        }
      }
    }
    const long long row = (long long)c.row0 + token, head = (long long)c.r * pd.g_q + m % pd.g_q;
    const float inv = reciprocal(sm);
    __nv_bfloat16* op = a.O + row * pd.os[0] + head * pd.os[1] + col;
#pragma unroll
    for (int q = 0; q < 8; q += 2)
      *reinterpret_cast<uint4*>(op + q * 4) = make_uint4(pack2(acc[q].x * inv, acc[q].y * inv), pack2(acc[q].z * inv, acc[q].w * inv),
                                                         pack2(acc[q + 1].x * inv, acc[q + 1].y * inv), pack2(acc[q + 1].z * inv, acc[q + 1].w * inv));
    if (col == 0 && a.lse) a.lse[row * pd.h_q + head] = lse_of(mx, sm);
    return;
  }
  const int rows = c.tokens * pd.g_q;
  int span = 128;                             // the rows, up to a power of two; R of them are a share
  while (span > 1 && span / 2 >= rows) span >>= 1;
  const int R = max(1, span / JOIN_SHARES), row0 = blockIdx.y * R;
  if (row0 >= rows) return;
  const int parts = 2 * c.blocks, work = R * C4, P = JOIN_THREADS / work;
  {
    const int mine = tid / work, w = tid - mine * work, r = w & (R - 1), piece = w / R, m = row0 + r;
    float mx = -INFINITY, sm = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m < rows) {
#pragma unroll 8
      for (int k = mine; k < parts; k += P) {
        const float* part = partial_at<HD>(a, first + (k >> 1), k < 2 ? 1 : 0, k & 1);
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(part + 128 * HD) + m);
        const float4 x = __ldcg(reinterpret_cast<const float4*>(part) + piece * 128 + m);
        if (ml.x != -INFINITY) {
          const float top = max2(mx, ml.x), corr = exp2f(mx - top), wt = exp2f(ml.x - top);
          mx = top;
          sm = fmaf(ml.y, wt, sm * corr);
          acc.x = fmaf(x.x, wt, acc.x * corr); acc.y = fmaf(x.y, wt, acc.y * corr);
          acc.z = fmaf(x.z, wt, acc.z * corr); acc.w = fmaf(x.w, wt, acc.w * corr);
        }
      }
    }
    out[(mine * R + r) * C4 + piece] = acc;
    if (piece == 0) stat[mine * R + r] = make_float2(mx, sm);
  }
  __syncthreads();
  for (int e = tid; e < R * (HD / 8); e += JOIN_THREADS) {
    const int r = e / (HD / 8), q = e - r * (HD / 8), m = row0 + r;
    if (m >= rows) continue;
    float top = -INFINITY, l = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
    for (int k = 0; k < P; ++k) top = max2(top, stat[k * R + r].x);
    for (int k = 0; k < P; ++k) {
      const float2 ml = stat[k * R + r];
      if (ml.x == -INFINITY) continue;
      const float wt = exp2f(ml.x - top);
      const float4 u = out[(k * R + r) * C4 + 2 * q], v = out[(k * R + r) * C4 + 2 * q + 1];
      l = fmaf(ml.y, wt, l);
      x.x = fmaf(u.x, wt, x.x); x.y = fmaf(u.y, wt, x.y); x.z = fmaf(u.z, wt, x.z); x.w = fmaf(u.w, wt, x.w);
      y.x = fmaf(v.x, wt, y.x); y.y = fmaf(v.y, wt, y.y); y.z = fmaf(v.z, wt, y.z); y.w = fmaf(v.w, wt, y.w);
    }
    const float inv = reciprocal(l);
    const long long row = (long long)c.row0 + m / pd.g_q, head = (long long)c.r * pd.g_q + m % pd.g_q;
    *reinterpret_cast<uint4*>(a.O + row * pd.os[0] + head * pd.os[1] + q * 8) =
        make_uint4(pack2(x.x * inv, x.y * inv), pack2(x.z * inv, x.w * inv), pack2(y.x * inv, y.y * inv), pack2(y.z * inv, y.w * inv));
    if (q == 0 && a.lse) a.lse[row * pd.h_q + head] = lse_of(top, l);
  }
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
    // (the kernel uses a block per two tiles at most, and the tables bound their number)
    const long long most = (long long)a.n_slots * ((a.pd.cap + NT - 1) / NT) * a.pd.h_kv;
    const unsigned blocks = (unsigned)(most < 2LL * a.n_blocks ? (most + 1) / 2 : a.n_blocks);
    cudaError_t e = launch_chained(kern, dim3(blocks), dim3(THREADS), Layout<HD>::smem(a.n_slots), st, tq, tk, tv, a);
    count_launch();
    if (e != cudaSuccess) return e;
    if (a.pd.cap <= NT) continue;              // units of one tile are not cut
    e = launch_chained(chunk_join_kernel<HD>, dim3(blocks, JOIN_SHARES), dim3(JOIN_THREADS), 0, st, a);
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

// The cuts, then the blocks' partial results.
size_t chunk_sm100_partial_bytes(const PagedDims& pd) {
  const size_t floats = pd.d == 128 ? partial_floats<128>() : partial_floats<64>();
  return (size_t)current_sm_count() * (sizeof(Cut) + PARTS * floats * sizeof(float));
}

cudaError_t launch_attend_chunk_sm100(const PagedDims& pd, const void* Q, const void* Kpool, const void* Vpool,
                                      const int* page_table, const int* q_start, const int* kv_len, void* O, float* lse,
                                      float* partials, StatusBlock* sb, cudaStream_t st) {
  ChunkArgs a;
  a.pd = pd;
  a.TQ = 128 / pd.g_q;
  a.box = paged_box(pd);
  a.n_blocks = current_sm_count();
  a.q_start = q_start; a.kv_len = kv_len; a.page_table = page_table;
  a.O = (__nv_bfloat16*)O;
  a.lse = lse;
  a.cuts = reinterpret_cast<Cut*>(partials);
  a.partials = partials + (size_t)a.n_blocks * sizeof(Cut) / sizeof(float);
  a.sb = sb;
  a.hold = test_hooks().hold_cycles;
  a.hold_odd = test_hooks().hold_odd;
  a.inject = test_hooks().skip_own_k_load;
  a.wait_limit = test_hooks().wait_limit_cycles;
  CUtensorMap tq, tk, tv;
  if (!paged_q_map(&tq, pd, Q, a.TQ) || !paged_pool_map(&tk, pd, Kpool, pd.ks, a.box) || !paged_pool_map(&tv, pd, Vpool, pd.vs, a.box))
    return cudaErrorInvalidValue;
  return pd.d == 128 ? launch_hd<128>(a, tq, tk, tv, st) : launch_hd<64>(a, tq, tk, tv, st);
}

}  // namespace dash
