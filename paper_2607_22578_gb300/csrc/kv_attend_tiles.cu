// Attention of many query rows over the paged 8-bit cache (hs_kv_attend): prompts, chunks and
// cross attention, on the tensor cores.
//
// The formula is kv_attend.cu's.  A step is 128 rows (query, head of the group) against 128
// tokens: s = q k^T is one tcgen05.mma per 16 of dim (M = 128, N = 128) into tensor memory, o += p v
// one per 16 tokens (N = dim) with p as its A operand in tensor memory, where the scores were.  4
// flops a (row, token, dim) and one exponential a (row, token): tensor cores and exponentials bound
// it together, so a CTA keeps two tiles of rows in flight that take turns: while one's scores become
// weights, the tensor cores work for the other.  Scores become weights by halves of the tokens, each
// a step of the running maximum, and each half is handed over when it is done.
// (Two buffers of scores of 64 tokens each instead of one of 128: a product of N = 64 takes as long
// as one of 128, 75 clocks, and the whole 4700 clocks for 128 tokens instead of 4500.)
//
//   warps 0-3, 4-7   a thread a row: its query into shared memory, scores to weights, the output
//   warps 8-14       codes from the cache's blocks, decoded to half in shared memory (swizzled;
//                    K and V alike: K is read along dim, V across it), a tile ahead in registers
//   warp 15          one thread issues every product
//
// CTAs are persistent, one an SM.  Work is (request, pair of tiles of rows, kv head) items, longest
// requests first and the later pairs of a request (which see more) first, taken from a queue (a
// counter in the workspace, drawn from an item ahead): items are few and differ by much, and in a
// fixed order the two cases below take 378 and 485 us.  An item's queries and first
// tokens are loaded while the one before it ends.  Which CTA computes an item changes no result.
// Where there are fewer items than half the CTAs, an item's tokens are up to eight parts, each an item
// of its own; a warp's rows of the parts are merged by the one that is done last (128 queries over
// 16,384 tokens, 32 / 8 heads of 128: 313 -> 62 us).
//
// Measured: 16 prompts of 256 to 2048 tokens, 32 / 8 heads of 128, 343 us (610 TFLOP/s); six chunks of
// up to 1024 queries behind 1,000 to 12,000 tokens, 32 / 4 heads, 468 (710).  256 rows by 128 tokens
// take 4650 clocks, products 2200 of them: the rest is the chain of one tile (scores loaded, maxima,
// 64 exponentials and their factors a thread, twice, then the last product and the next scores).
//
// Arithmetic: q as half after division by a power of two of its row; codes as half (exact); sums
// in fp32.  With c a score's factor and vs the values' scale of its block, a row keeps two running
// maxima (both may lag by 8): ms of the scores s = acc * c, and m of s + log2 vs.  The weights' sum
// is of z = 2^(s - ms + 7), the output's weights are w = z * vs * 2^(ms - m) as half, o = sum w code,
// and o * 2^(m - ms) / sum is the output.  With one maximum for both, a block of zeros (scale 2^-126)
// would drop out of the sum, or overflow it; as it is, a weight is lost where it is below 2^-126 of
// the row's largest, whatever the scales are.  (The second maximum and the factors: prompts 329 -> 337 us,
// cross attention 52.4 -> 54.6.)
#include "kv_attend.cuh"
#include "kv_cache.cuh"

namespace hs {
namespace {

constexpr int kTileRows = 128;
constexpr int kPairRows = 2 * kTileRows;
constexpr int kTileTokens = 128;
constexpr int kGroups = kTileTokens / 16;      // 16 tokens lie in one block: one scale
constexpr int kSoftWarps = 8;
constexpr int kLoadWarp = 8;                   // the first of seven
constexpr int kLoadWarps = 7;
constexpr int kMmaWarp = 15;
constexpr int kTilesThreads = 16 * 32;
constexpr int kHalfTokens = kTileTokens / 2;
constexpr int kHalfGroups = kGroups / 2;
constexpr int kLoadThreads = kLoadWarps * 32;
constexpr int kScaleRing = 4;                  // tiles
constexpr int kItemRing = 4;
constexpr int kMostParts = 8;                  // of an item
constexpr int kLeastSteps = 4;                 // of a part
constexpr float kTilesLag = 8.0f;
constexpr float kTilesShift = 7.0f;
constexpr float kLeastScale = 1.17549435e-38f;
constexpr float kMostFactor = 8.5070592e37f;   // 2^126

template <int D>
struct TilesLayout {
  static constexpr int kBlockBytes = 128 * 128;              // 64 of dim, 128 rows
  static constexpr int kTileBytes = D / 64 * kBlockBytes;    // 128 rows or tokens of dim as half
  static constexpr int kQ = 0;                               // two tiles
  static constexpr int kK = 2 * kTileBytes;                  // two stages
  static constexpr int kV = 4 * kTileBytes;                  // two stages
  static constexpr int kOut = 6 * kTileBytes;                // 2 KB a warp: 32 rows, 32 of dim
  static constexpr int kEnd = kOut + kSoftWarps * 2048;
  static constexpr int kSmem = kEnd + 1024;                  // the base is aligned to 1024
};

struct Item {
  int32_t r, h, rows0, n, q0, len;
  int32_t tile0, tiles, rows;        // tiles of tokens; rows of the request
  int32_t steps0, steps1;            // of these for each tile of rows (0: it has no rows)
  int32_t more;                      // 0: no further item
  int32_t first;                     // token that a query sees
  // A part of the tokens: the first part's place among the partial results (16 bits), which part
  // it is (4), how many there are for each tile of rows (4, 4).
  uint32_t part;
};

// Partial results of a warp's 32 rows: both maxima, sums, outputs (four of dim of each row, then the
// next)
template <int D>
constexpr int64_t part_floats() { return 32 * (D + 3); }

// Whether a phase is over, without waiting (try_wait may sleep until it is)
__device__ __forceinline__ bool test_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

// The wait of kWaitLimitNs, out of line: the instruction cache is small beside this kernel.
__device__ __noinline__ bool wait_on(uint32_t bar, uint32_t parity, volatile int* abort) {
  const uint64_t t0 = globaltimer_ns();
  for (uint32_t it = 1;; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 63u) == 0) {
      if (*abort) return false;
      if (globaltimer_ns() - t0 > kWaitLimitNs) {
        *abort = 1;
        return false;
      }
    }
  }
}

struct TilesShared {
  uint64_t item_full[kItemRing], item_empty[kItemRing];
  uint64_t q_full[2];
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t s_full[2];                   // of a tile of rows
  uint64_t p_full[2][2], o_full[2][2];  // ... and half of the tokens
  uint64_t drained;
  Item items[kItemRing];
  int4 outputs[kSoftWarps];             // what a warp's output needs of its item (registers are few):
                                        // its tile's first row, rows, the place of row 0, its parts
  // of 16 tokens: keys', log2 of values' (always a number), values'; NaN for what is no number
  float4 scales[kScaleRing][kGroups];
  uint32_t tmem;
  int abort;
  int32_t sums[kTilesThreads / 32];
  int32_t before[kTilesThreads + 1];    // items before each thread's requests
  int32_t order[kTilesThreads];         // up to that many requests, by length
  int32_t length[kTilesThreads], count[kTilesThreads];
};

__device__ __forceinline__ void fence_async_shared() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// D[tmem] (+)= A * B^T in half with fp32 sums: A in shared memory, or in tensor memory.
__device__ __forceinline__ void umma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                        uint32_t accumulate) {
  umma_bf16(d, a, b, idesc, accumulate);  // the types are idesc's
}
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a_tmem, uint64_t b, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void tmem_st_32x32b_x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// Instruction descriptor, kind::f16: D fp32, A and B half, A K-major, B K- or MN-major.
constexpr uint32_t idesc_f16(int M, int N, bool b_mn) {
  return (1u << 4) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) |
         ((uint32_t)(M >> 4) << 24);
}

// Shared-memory descriptor of an MN-major operand with 128-byte swizzling: rows of K, 64 of MN
// (128 bytes) each, 8 rows an atom (stride byte offset 1024), the next 64 of MN `lbo` bytes on.
__device__ __forceinline__ uint64_t smem_desc_mn_sw128(uint32_t saddr, uint32_t lbo) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(lbo >> 4) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= (uint64_t)1u << 46;
  d |= (uint64_t)2u << 61;
  return d;
}

// One thread of a converged warp, the same each time.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(p));
  return p != 0;
}

// Two floats at once (sm_100's packed fp32 operations)
__device__ __forceinline__ uint64_t pack_b32x2(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ uint64_t pack_f32x2(float lo, float hi) {
  return pack_b32x2(__float_as_uint(lo), __float_as_uint(hi));
}
__device__ __forceinline__ void unpack_f32x2(uint64_t v, float& lo, float& hi) {
  uint32_t a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(v));
  lo = __uint_as_float(a);
  hi = __uint_as_float(b);
}
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// The scores' factor; never 0, so that a hidden score's -inf stays one.
__device__ __forceinline__ float factor(float scale, float q_scale) {
  const float f = scale * q_scale;
  return f < kLeastScale ? kLeastScale : f;
}

__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}

struct Merged {
  float ms, m, sum;
  bool last;
};

// A warp's 32 rows of one part of an item: maxima and sums, outputs in tensor memory.  All but the
// part that is done last only leave them in memory; that one merges all of them, in the order of the
// parts, into its own place.  Out of line, for the same reason as wait_on.
template <int D>
__device__ __noinline__ Merged merge_parts(float* partial, unsigned* counters, uint32_t code,
                                           int32_t n_parts, uint32_t t_o, float ms, float m,
                                           float sum) {
  const int lane = threadIdx.x & 31;
  const int32_t at = (int32_t)(code & 0xffff) * kSoftWarps + (threadIdx.x >> 5);
  constexpr int64_t kNext = kSoftWarps * part_floats<D>();  // on to the next part
  float* all = partial + at * part_floats<D>();
  float* mine = all + ((code >> 16) & 15) * kNext;
  mine[lane] = m;
  mine[32 + lane] = sum;
  mine[64 + lane] = ms;
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    uint32_t o[32];
    tmem_ld_32x32b_x32(t_o + c * 32, o);
    tmem_ld_wait();
#pragma unroll
    for (int v = 0; v < 8; ++v)
      *reinterpret_cast<uint4*>(mine + 96 + ((c * 8 + v) * 32 + lane) * 4) =
          make_uint4(o[v * 4], o[v * 4 + 1], o[v * 4 + 2], o[v * 4 + 3]);
  }
  __threadfence();
  __syncwarp();
  uint32_t done = 0;
  if (lane == 0) {
    done = atomicAdd(counters + at, 1u) + 1;
    if ((int32_t)done == n_parts) counters[at] = 0;  // as the next call finds it
    __threadfence();
  }
  Merged r{ms, m, sum, (int32_t)__shfl_sync(0xffffffffu, done, 0) == n_parts};
  if (!r.last) return r;
  // the parts' factors: of sums by the scores' maxima, then of outputs by the others
  float w[kMostParts];
  r.sum = 0.0f;
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    float now = -INFINITY;
#pragma unroll
    for (int k = 0; k < kMostParts; ++k) {
      w[k] = k < n_parts ? __ldcg(all + k * kNext + (y ? 0 : 64) + lane) : -INFINITY;
      now = fmaxf(now, w[k]);
    }
#pragma unroll
    for (int k = 0; k < kMostParts; ++k) {
      w[k] = w[k] == -INFINITY ? 0.0f : fast_exp2(w[k] - now);
      if (y == 0 && k < n_parts) r.sum = fmaf(w[k], __ldcg(all + k * kNext + 32 + lane), r.sum);
    }
    (y ? r.m : r.ms) = now;
  }
#pragma unroll 1
  for (int c = 0; c < D / 16; ++c) {
    const float4* from = reinterpret_cast<const float4*>(all + 96) + c * 4 * 32 + lane;
    float o[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] = 0.0f;
#pragma unroll
    for (int k = 0; k < kMostParts; ++k) {
      if (k < n_parts) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float4 y = __ldcg(from + k * (kNext / 4) + v * 32);
          o[v * 4] = fmaf(w[k], y.x, o[v * 4]);
          o[v * 4 + 1] = fmaf(w[k], y.y, o[v * 4 + 1]);
          o[v * 4 + 2] = fmaf(w[k], y.z, o[v * 4 + 2]);
          o[v * 4 + 3] = fmaf(w[k], y.w, o[v * 4 + 3]);
        }
      }
    }
    tmem_st_32x32b_x16(t_o + c * 16, reinterpret_cast<uint32_t(&)[16]>(o));
  }
  tmem_st_wait();
  return r;
}

// Pairs of row tiles of request r (0: none, or another kernel's).
__device__ __forceinline__ int32_t request_pairs(const AttendParams& p, int32_t r, Item& it,
                                                 unsigned* bad) {
  if (!attend_request(p, r, it.n, it.q0, it.len, bad)) return 0;
  it.rows = it.n * p.G;
  if (it.rows <= p.rows_most) return 0;
  return (it.rows + kPairRows - 1) / kPairRows;
}

template <int D, int FMT>
__global__ void __launch_bounds__(kTilesThreads, 1) kv_attend_tiles_kernel(const AttendParams p) {
  using L = TilesLayout<D>;
  extern __shared__ uint8_t raw[];
  __shared__ TilesShared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;

  if (tid == 0) {
    for (int i = 0; i < kItemRing; ++i) {
      mbar_init(&sh.item_full[i], 1);
      mbar_init(&sh.item_empty[i], kSoftWarps + 1 + kLoadWarps - 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], kTileRows);
      mbar_init(&sh.k_full[i], kLoadThreads);
      mbar_init(&sh.k_empty[i], 1);
      mbar_init(&sh.v_full[i], kLoadThreads);
      mbar_init(&sh.v_empty[i], 1);
      mbar_init(&sh.s_full[i], 2);
      for (int j = 0; j < 2; ++j) {
        mbar_init(&sh.p_full[i][j], kTileRows);
        mbar_init(&sh.o_full[i][j], 1);
      }
    }
    mbar_init(&sh.drained, 1);
    fence_mbar_init();
    sh.abort = 0;
  }
  if (warp == kMmaWarp) {
    tmem_alloc(&sh.tmem, 512);
    tmem_relinquish();
  }
  pdl_wait();
  pdl_trigger();
  const int32_t R = p.n_req_dev ? max(0, min(__ldg(p.n_req_dev), p.n_req)) : p.n_req;

  // ---- items before each thread's requests
  unsigned bad = 0;
  const int32_t per = (R + kTilesThreads - 1) / kTilesThreads;
  {
    const int32_t ra = min(tid * per, R), rb = min(ra + per, R);
    int32_t mine = 0;
    Item it{};
#pragma unroll 1
    for (int32_t r = ra; r < rb; ++r) mine += request_pairs(p, r, it, &bad);
    if (per <= 1) {                               // a request a thread: in the order of their lengths
      if (tid < R) sh.length[tid] = mine ? it.len : -1;
      __syncthreads();
      if (tid < R) {
        const int32_t len = sh.length[tid];
        int32_t rank = 0;
#pragma unroll 4
        for (int32_t r = 0; r < R; ++r) {
          const int32_t other = sh.length[r];
          rank += other > len || (other == len && r < tid);
        }
        sh.order[rank] = tid;
        sh.count[rank] = mine;
      }
      __syncthreads();
      mine = tid < R ? sh.count[tid] : 0;
    }
    mine *= p.H;
    int32_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    if (lane == 31) sh.sums[warp] = incl;
    __syncthreads();
    int32_t b = 0;
    for (int w = 0; w < warp; ++w) b += sh.sums[w];
    sh.before[tid] = b + incl - mine;
    if (tid == kTilesThreads - 1) sh.before[kTilesThreads] = b + incl;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (bad && blockIdx.x == 0) set_error(p.err, bad);
  // Fewer items than CTAs: the tokens of each in parts, whose results the last to be done merges.
  const int32_t whole = sh.before[kTilesThreads];
  const int32_t parts = min(kMostParts, max(1, (int32_t)gridDim.x / max(1, whole)));
  const int32_t total = whole * parts;
  const uint32_t tmem = sh.tmem;
  volatile int* abort = &sh.abort;
  const auto wait = [&](uint64_t* bar, uint32_t phase) {  // a warp goes on, or gives up, as one
    const uint32_t a = smem_u32(bar);
    return __all_sync(0xffffffffu, mbar_try_wait(a, phase & 1u) || wait_on(a, phase & 1u, abort)) != 0;
  };

  if (warp >= kLoadWarp && warp < kMmaWarp) {
    // ================================ keys and values
    const int lw = warp - kLoadWarp;
    const int row8 = lane & 7, chunk = lane >> 3;   // of 8 tokens' 64 bytes
    constexpr int RG = (kTileTokens / 8 + kLoadWarps - 1) / kLoadWarps;  // groups of 8 tokens, mine
    constexpr int CH = D / 64;

    // The tiles of this CTA's items end to end: of the one whose blocks were looked up last, its
    // item, and its blocks, place and length, for the loads to come.
    Item it{};
    int32_t at = blockIdx.x, tile = 0;              // the next item, and tile of `it`
    int32_t drawn = 0;                              // ... and the one after, for the first warp
    const auto draw = [&]() {
      if (lw == 0 && lane == 0) drawn = (int32_t)(gridDim.x + atomicAdd(p.queue, 1u));
    };
    draw();
    uint32_t items = 0;                             // said so far
    bool ok = true;
    int32_t ids[RG], sid = -1, t_len = 0, t_first = 0, t_h = 0, t_0 = 0;
    const auto look_up = [&]() {                    // false: there is no further tile
      if (tile == it.tile0 + it.tiles) {            // the next item, for everybody
        const uint32_t slot = items & (kItemRing - 1);
        if (lw > 0) {                               // as the first warp says
          if (!(ok = wait(&sh.item_full[slot], items / kItemRing))) return false;
          it = sh.items[slot];
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.item_empty[slot]);
        } else {
          it = Item{};
          do {
            it.more = at < total;
            if (!it.more) break;
            const int32_t of = parts > 1 ? at / parts : at, part = at - of * parts;
            int lo = 0, hi = kTilesThreads;           // the last thread with before <= of
#pragma unroll 1
            while (hi - lo > 1) {
              const int mid = (lo + hi) >> 1;
              if (sh.before[mid] <= of) lo = mid; else hi = mid;
            }
            int32_t x = of - sh.before[lo], pairs = 0;
            int32_t r = per <= 1 ? sh.order[lo] : lo * per;
#pragma unroll 1
            for (;; ++r) {
              pairs = request_pairs(p, r, it, &bad);
              if (per <= 1 || x < pairs * p.H || r + 1 >= min((lo + 1) * per, R)) break;
              x -= pairs * p.H;
            }
            const int32_t back = x / p.H;
            it.r = r;
            it.h = x - back * p.H;
            it.rows0 = max(pairs - 1 - back, 0) * kPairRows;
            const int32_t before_q = it.len - it.n;   // the first query's position
            it.first = attend_first(p, it.n, it.len);
            it.tile0 = p.window > 0
                           ? max(0, before_q + attend_query(p, it.rows0) - attend_window(p, it.len) +
                                        1) / kTileTokens
                           : 0;
            const auto steps = [&](int32_t first) {   // of the tile of rows that begins there
              if (first >= it.rows) return 0;
              const int32_t i1 = min(it.n - 1, attend_query(p, first + kTileRows - 1));
              const int32_t see = p.causal ? min(it.len, before_q + i1 + 1) : it.len;
              // (where nothing is seen: one, hidden)
              return max(1, (see + kTileTokens - 1) / kTileTokens - it.tile0);
            };
            it.steps0 = steps(it.rows0);
            it.steps1 = steps(it.rows0 + kTileRows);
            it.tiles = max(it.steps0, it.steps1);
            if (parts > 1) {
              const int32_t each = max(kLeastSteps, (it.tiles + parts - 1) / parts);
              it.part = (uint32_t)(of * parts) | (uint32_t)part << 16 |
                        (uint32_t)((it.steps0 + each - 1) / each) << 20 |
                        (uint32_t)((it.steps1 + each - 1) / each) << 24;
              it.steps0 = min(max(it.steps0 - part * each, 0), each);
              it.steps1 = min(max(it.steps1 - part * each, 0), each);
              it.tiles = max(it.steps0, it.steps1);
              it.tile0 += part * each;
            }
            at = __shfl_sync(0xffffffffu, drawn, 0);
            if (at < total) draw();
          } while (it.tiles == 0);                    // (fewer parts than the others have)
          if (items >= kItemRing) ok = wait(&sh.item_empty[slot], items / kItemRing - 1);
          if (lw == 0 && lane == 0 && ok) {
            sh.items[slot] = it;
            mbar_arrive(&sh.item_full[slot]);
          }
        }
        ++items;
        tile = it.tile0;
        if (!ok || !it.more) return false;
      }
      t_len = it.len;
      t_first = it.first;
      t_h = it.h;
      t_0 = tile++ * kTileTokens;
      const int32_t* row = p.table + (int64_t)it.r * p.width;
#pragma unroll
      for (int i = 0; i < RG; ++i) {
        const int32_t g = lw + i * kLoadWarps, tok = t_0 + g * 8;
        ids[i] = g < kTileTokens / 8 && tok < t_len ? __ldg(row + (tok >> p.bt_log2)) : -1;
      }
      if (lw == 0 && lane < kGroups)
        sid = t_0 + lane * 16 < t_len ? __ldg(row + ((t_0 + lane * 16) >> p.bt_log2)) : -1;
      return true;
    };
    uint4 kr[RG][CH], vr[RG][CH];
    int64_t off[RG];                                // of this thread's 16 bytes; -1: no token
    float2 scale = make_float2(0.0f, 0.0f);         // of 16 tokens, for this lane
    const auto fetch = [&](const uint8_t* codes, uint4 (&to)[RG][CH]) {
#pragma unroll
      for (int i = 0; i < RG; ++i)
#pragma unroll
        for (int c = 0; c < CH; ++c)
          to[i][c] = off[i] >= 0 ? __ldg(reinterpret_cast<const uint4*>(codes + off[i] + c * 64))
                                 : make_uint4(0u, 0u, 0u, 0u);
    };
    const auto put = [&](uint32_t to, const uint4 (&from)[RG][CH]) {
#pragma unroll
      for (int i = 0; i < RG; ++i) {
        const int g = lw + i * kLoadWarps;
        if (g >= kTileTokens / 8) break;
        const int row = g * 8 + row8;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const uint32_t w[4] = {from[i][c].x, from[i][c].y, from[i][c].z, from[i][c].w};
          uint32_t h[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            h[2 * e] = KvFormat<FMT>::template decode2<0>(w[e]);
            h[2 * e + 1] = KvFormat<FMT>::template decode2<1>(w[e]);
          }
          const uint32_t line = to + c * L::kBlockBytes + row * 128;
          sts128(line + (((2 * chunk) ^ row8) << 4), h[0], h[1], h[2], h[3]);
          sts128(line + (((2 * chunk + 1) ^ row8) << 4), h[4], h[5], h[6], h[7]);
        }
      }
    };
    // Round n lays out tile n - 1 and fetches tile n into the registers that get free.
    bool looked = look_up(), fetched = false;
#pragma unroll 1
    for (uint32_t n = 0; ok && (looked || fetched); ++n) {
      const uint32_t st = (n - 1) & 1, use = (n - 1) >> 1;
      if (fetched) {
        if (n > 2 && !(ok = wait(&sh.k_empty[st], use - 1))) break;
        if (lw == 0 && lane < kGroups) {
          const bool k = scale.x < INFINITY, v = scale.y < INFINITY;    // (a NaN is not)
          sh.scales[(n - 1) & (kScaleRing - 1)][lane] =
              make_float4(k ? fmaxf(scale.x, kLeastScale) : __int_as_float(0x7fffffff),
                          v ? log2f(fmaxf(scale.y, kLeastScale)) : 0.0f,
                          v ? scale.y : __int_as_float(0x7fffffff), 0.0f);
        }
        put(base + L::kK + st * L::kTileBytes, kr);
        fence_async_shared();
        mbar_arrive(&sh.k_full[st]);
      }
      if (looked) {
#pragma unroll
        for (int i = 0; i < RG; ++i) {
          const int32_t tok = t_0 + (lw + i * kLoadWarps) * 8 + row8, id = ids[i];
          const bool known = (uint32_t)id < (uint32_t)p.n_blocks;
          if (id != -1 && !known) bad = kErrInvalidArg;
          off[i] = known && tok < t_len && tok >= t_first
                       ? ((((int64_t)id * p.H + t_h) << p.bt_log2) +
                          (tok & ((1 << p.bt_log2) - 1))) * D + chunk * 16
                       : -1;
        }
        fetch(p.k, kr);
        if (lw == 0 && lane < kGroups) {
          const bool in = (uint32_t)sid < (uint32_t)p.n_blocks;
          if (!in && t_0 + lane * 16 < t_len) bad = kErrInvalidArg;
          scale.x = in ? __ldg(p.ks + (int64_t)sid * p.H + t_h) : 0.0f;
          scale.y = in ? __ldg(p.vs + (int64_t)sid * p.H + t_h) : 0.0f;
        }
      }
      if (fetched) {
        if (n > 2 && !(ok = wait(&sh.v_empty[st], use - 1))) break;
        put(base + L::kV + st * L::kTileBytes, vr);
        fence_async_shared();
        mbar_arrive(&sh.v_full[st]);
      }
      if (looked) fetch(p.v, vr);
      fetched = looked;
      if (looked) looked = look_up();
    }
    // The last CTA to be done with the queue leaves it as the next call finds it.
    if (lw == 0 && lane == 0) {
      __threadfence();                              // its draws come before
      if (atomicAdd(p.queue + 1, 1u) == gridDim.x - 1) {
        p.queue[0] = 0;
        p.queue[1] = 0;
      }
    }
  } else if (warp == kMmaWarp) {
    // ================================ products
    // The whole warp runs this, so that descriptors stay in uniform registers; one thread issues.
    {
      constexpr uint32_t id_qk = idesc_f16(kTileRows, kTileTokens, false);
      constexpr uint32_t id_pv = idesc_f16(kTileRows, D, true);
      const uint64_t d_q = smem_desc_k_sw128(base + L::kQ);
      const uint64_t d_k = smem_desc_k_sw128(base + L::kK);
      const uint64_t d_v = smem_desc_mn_sw128(base + L::kV, L::kBlockBytes);
      const auto qk = [&](int x, uint32_t st) {
        const uint64_t a = d_q + (x * L::kTileBytes >> 4), b = d_k + (st * L::kTileBytes >> 4);
        const uint32_t to = tmem + x * kTileTokens;
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const int off = ((k >> 2) * L::kBlockBytes + (k & 3) * 32) >> 4;
            umma_ss(to, a + off, b + off, id_qk, k > 0);
          }
          umma_commit(&sh.s_full[x]);
          mbar_arrive(&sh.s_full[x]);                 // passes on what this thread has seen: the scales
        }
        __syncwarp();
      };
      const auto pv = [&](int x, uint32_t st, int half, bool add) {
        const uint64_t b = d_v + (st * L::kTileBytes >> 4);
        const uint32_t to = tmem + 2 * kTileTokens + x * D, from = tmem + x * kTileTokens;
        if (elect_one()) {
#pragma unroll
          for (int i = 0; i < kTileTokens / 32; ++i) {
            const int k = half * (kTileTokens / 32) + i;
            umma_ts(to, from + k * 8, b + (k * 2048 >> 4), id_pv, k > 0 ? 1u : add);
          }
          umma_commit(&sh.o_full[x][half]);
        }
        __syncwarp();
      };
      const auto commit = [&](uint64_t* bar) {
        if (elect_one()) umma_commit(bar);
        __syncwarp();
      };
      uint32_t tiles = 0, ns[2] = {0, 0}, nq[2] = {0, 0};  // of the CTA; steps, items of each tile of rows
      bool ok = true;
      for (uint32_t items = 0; ok; ++items) {
        const uint32_t slot = items & (kItemRing - 1);
        if (!(ok = wait(&sh.item_full[slot], items / kItemRing))) break;
        const int32_t s0 = sh.items[slot].steps0, s1 = sh.items[slot].steps1;
        const int32_t steps = max(s0, s1);
        if (!sh.items[slot].more) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.item_empty[slot]);
        // Step u's scores come after step u - 1's output, which read weights from their place.
        for (int32_t u = 0; u <= steps && ok; ++u) {
          const uint32_t tile = tiles + u, st = tile & 1;
          if (u < steps) {
            if (!(ok = wait(&sh.k_full[st], tile >> 1))) break;
            tc_fence_after();
          }
          const auto turn = [&](int x, int32_t mine) {
            if (u > 0 && u <= mine) {
              const uint32_t sv = st ^ 1;
              if (x == 0 || s0 < u)                    // the first to read these values
                if (!(ok = wait(&sh.v_full[sv], (tile - 1) >> 1))) return;
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                if (!(ok = wait(&sh.p_full[x][half], ns[x]))) return;
                tc_fence_after();
                pv(x, sv, half, u > 1);
              }
              ++ns[x];
            }
            if (u < mine) {
              if (u == 0) {
                if (!(ok = wait(&sh.q_full[x], nq[x]++))) return;
                tc_fence_after();
              }
              qk(x, st);
            }
          };
          turn(0, s0);
          if (!ok) break;
          if (s1 > 0) turn(1, s1);
          if (!ok) break;
          if (u > 0) commit(&sh.v_empty[st ^ 1]);
          if (u < steps) commit(&sh.k_empty[st]);
        }
        tiles += steps;
      }
      commit(&sh.drained);                     // nothing of it runs on when memory is given back
      if (!mbar_wait_limit(&sh.drained, 0, abort, kWaitLimitNs)) {
        const uint64_t t0 = globaltimer_ns();       // someone gave up: wait for what was issued
        while (!mbar_try_wait(smem_u32(&sh.drained), 0) && globaltimer_ns() - t0 < kWaitLimitNs) {
        }
      }
    }
    __syncwarp();
  } else {
    // ================================ queries, scores to weights, the output
    const int x = warp >> 2;                        // which tile of rows
    const int row = (warp & 3) * 32 + lane;         // of it, and lane of tensor memory
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + x * kTileTokens;
    const uint32_t t_o = tmem + lanes + 2 * kTileTokens + x * D;
    uint32_t items = 0, tiles = 0, ns = 0;          // of the CTA; steps of this tile of rows
    bool ok = true;

    // Queries: D / 8 lanes a row, 8 values each, so that a load is of whole rows.  They are copied to
    // their place as they are, while the last step's scores become weights, and become half there.
    constexpr int LR = D / 8, RS = 32 / LR, NQ = 32 / RS;  // lanes of a row, rows of a load, loads
    // The next item with rows of this tile's, if it has been said: the items up to it may have to
    // be done first, and they may need the step that this tile of rows is at.
    bool more = false;
    const auto take = [&](bool block) {
      for (;;) {
        const uint32_t slot = items & (kItemRing - 1), phase = items / kItemRing;
        if (block) {
          if (!(ok = wait(&sh.item_full[slot], phase))) return false;
        } else if (!__all_sync(0xffffffffu,
                               test_wait(smem_u32(&sh.item_full[slot]), phase & 1u))) {
          return false;
        }
        const Item& next = sh.items[slot];
        more = next.more != 0;
        if (!more || (x ? next.steps1 : next.steps0) > 0) return true;
        tiles += next.tiles;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.item_empty[slot]);
        ++items;
      }
    };
    const int q_row = (warp & 3) * 32 + lane / LR, q_chunk = lane % LR;  // of this thread's first load
    const uint32_t q_line = base + L::kQ + x * L::kTileBytes + (q_chunk >> 3) * L::kBlockBytes;
    const auto q_place = [&](int i) {
      const int r = q_row + i * RS;
      return q_line + r * 128 + (((q_chunk ^ r) & 7) << 4);
    };
    const auto fetch = [&]() {
      const Item& next = sh.items[items & (kItemRing - 1)];
      const int32_t first = next.rows0 + x * kTileRows + q_row, rows = next.rows;
      const uint16_t* src = p.q + (int64_t)next.q0 * p.q_token +
                            (int64_t)(next.h * p.G) * p.q_head + q_chunk * 8;
      const int64_t wrap = p.q_token - (int64_t)p.G * p.q_head;  // on to the next query
#pragma unroll 1
      for (int i = 0; i < NQ; ++i) {
        const int32_t full = first + i * RS;
        const bool in = full < rows;
        const int32_t at = in ? full : 0;
        const uint16_t* from = src + attend_query(p, at) * wrap + at * p.q_head;
        if (p.q_vec) {
          cp_async16_zfill(q_place(i), from, in);
        } else {
          const uint4 v = in ? attend_raw8(from) : make_uint4(0u, 0u, 0u, 0u);
          sts128(q_place(i), v.x, v.y, v.z, v.w);
        }
      }
    };
    float qs = 0.0f;
    const auto put = [&]() {                        // a thread has a row, in place
      cp_async_wait_all();
      __syncwarp();
      const uint32_t line = base + L::kQ + x * L::kTileBytes + row * 128;
      uint32_t bits = 0;                            // the row's largest, as in 16 bits without a sign
      uint4 v[LR];
#pragma unroll
      for (int ch = 0; ch < LR; ++ch) {
        v[ch] = lds128(line + (ch >> 3) * L::kBlockBytes + (((ch ^ row) & 7) << 4));
        const uint32_t w[4] = {v[ch].x, v[ch].y, v[ch].z, v[ch].w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          asm("max.u16x2 %0, %0, %1;" : "+r"(bits) : "r"(w[e] & 0x7fff7fffu));
      }
      const float2 big = attend_unpack2(bits, p.fp16);
      // a power of two of the row's size, kept where it and its inverse are normal
      const uint32_t e = min(max(__float_as_uint(fmaxf(big.x, big.y)) >> 23, 1u), 253u);
      const float by = __uint_as_float((254u - e) << 23);
#pragma unroll
      for (int ch = 0; ch < LR; ++ch) {
        float f[8];
        attend_unpack8(v[ch], p.fp16, f);
        sts128(line + (ch >> 3) * L::kBlockBytes + (((ch ^ row) & 7) << 4),
               half2_of(f[0] * by, f[1] * by), half2_of(f[2] * by, f[3] * by),
               half2_of(f[4] * by, f[5] * by), half2_of(f[6] * by, f[7] * by));
      }
      qs = __uint_as_float(e << 23) * p.scale_log2;
      fence_async_shared();
      mbar_arrive(&sh.q_full[x]);
    };
    bool known = false, started = false;
    float ms = -INFINITY, m = -INFINITY, sum = 0.0f;
    for (;;) {
      if (!known) {
        if (!take(true)) break;
        if (more) fetch();
      }
      if (more) put();

      if (started) {
        // ---- the output of the item before
        if (!(ok = wait(&sh.o_full[x][1], ns - 1))) break;
        tc_fence_after();
        __syncwarp();
        const int4 it = sh.outputs[warp];
        const int32_t rows0 = it.x, rows = it.y;
        const uint32_t part = (uint32_t)it.w;
        const auto output_row = [&](int32_t full) {
          const int32_t i = attend_query(p, full);
          return it.z + i * (p.H * p.G - p.G) + full;  // (the host has seen that 31 bits hold it)
        };
        const int32_t n_parts = (part >> (x ? 24 : 20)) & 15;
        bool last = true;
        if (n_parts > 1) {
          const Merged all = merge_parts<D>(p.tile_partial, p.tile_counters, part, n_parts,
                                            t_o, ms, m, sum);
          ms = all.ms;
          m = all.m;
          sum = all.sum;
          last = all.last;
        }
        if (last) {
          const bool none = sum == 0.0f;
          // 2^(m - ms) / sum in two factors, which are in range where the output is
          const float back = none ? 0.0f : fast_exp2(0.5f * (m - ms));
          const float inv = none ? 0.0f : __fdividef(back, sum);
          if (p.lse && rows0 + row < rows)
            p.lse[output_row(rows0 + row)] =
                none ? -INFINITY : (ms - kTilesShift + log2f(sum)) * 0.69314718055994531f;
          // 32 of dim at a time through shared memory: a thread has a row, a store 64 bytes of eight
          const uint32_t stage = base + L::kOut + warp * 2048;
          uint16_t* dst[4];
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int32_t full = rows0 + (warp & 3) * 32 + v * 8 + (lane >> 2);
            dst[v] =
                full < rows ? p.out + (int64_t)output_row(full) * D + (lane & 3) * 8 : nullptr;
          }
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_ld_32x32b_x32(t_o + c * 32, o);
            tmem_ld_wait();
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              uint32_t w[4];
#pragma unroll
              for (int e = 0; e < 4; ++e)
                w[e] = none ? 0u
                            : attend_pack2(p.fp16, __uint_as_float(o[v * 8 + 2 * e]) * inv * back,
                                           __uint_as_float(o[v * 8 + 2 * e + 1]) * inv * back);
              sts128(stage + lane * 64 + ((v ^ ((lane >> 1) & 3)) << 4), w[0], w[1], w[2], w[3]);
            }
            __syncwarp();
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int r = v * 8 + (lane >> 2);
              const uint4 y = lds128(stage + r * 64 + (((lane & 3) ^ ((r >> 1) & 3)) << 4));
              if (dst[v]) *reinterpret_cast<uint4*>(dst[v] + c * 32) = y;
            }
            __syncwarp();
          }
        }
        tc_fence_before();
      }
      if (!more) break;
      const uint32_t slot = items++ & (kItemRing - 1);
      const Item it = sh.items[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.item_empty[slot]);
      started = true;
      known = false;
      const int32_t n_steps = x ? it.steps1 : it.steps0;
      const int32_t rows0 = it.rows0 + x * kTileRows;
      if (lane == 0)
        sh.outputs[warp] =
            make_int4(rows0, it.rows, it.q0 * (p.H * p.G) + it.h * p.G, (int32_t)it.part);
      const int32_t pos = it.len - it.n + attend_query(p, min(rows0 + row, it.rows - 1));
      const int32_t top = p.causal ? min(pos, it.len - 1) : it.len - 1;
      const int32_t bottom = p.window > 0 ? pos - attend_window(p, it.len) + 1 : 0;
      // tokens that every row of the tile sees: from .. to
      const int32_t pos0 = it.len - it.n + attend_query(p, rows0);
      const int32_t pos1 = it.len - it.n + min(it.n - 1, attend_query(p, rows0 + kTileRows - 1));
      const int32_t to = p.causal ? min(pos0, it.len - 1) : it.len - 1;
      const int32_t from = p.window > 0 ? pos1 - attend_window(p, it.len) + 1 : 0;
      const uint32_t tile_base = tiles;
      tiles += it.tiles;

      ms = m = -INFINITY;
      sum = 0.0f;
      for (int32_t u = 0; u < n_steps; ++u, ++ns) {
        if (!(ok = wait(&sh.s_full[x], ns))) break;
        tc_fence_after();
        if (u + 1 == n_steps) {                       // the last product to read the queries is done
          known = take(false);
          if (known && more) fetch();
        }
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          const float4* scales =
              sh.scales[(tile_base + u) & (kScaleRing - 1)] + half * kHalfGroups;
          const int32_t t0 = (it.tile0 + u) * kTileTokens + half * kHalfTokens;
          uint32_t a[kHalfTokens];
          tmem_ld_32x32b_x32(t_s + half * kHalfTokens, *reinterpret_cast<uint32_t(*)[32]>(a));
          tmem_ld_32x32b_x32(t_s + half * kHalfTokens + 32,
                             *reinterpret_cast<uint32_t(*)[32]>(a + 32));
          float by[kHalfGroups], lv[kHalfGroups];
#pragma unroll
          for (int g = 0; g < kHalfGroups; ++g) {
            by[g] = factor(scales[g].x, qs);
            lv[g] = scales[g].y;
          }
          tmem_ld_wait();
          uint32_t hidden = 0;                        // groups of which this row sees no token
          if (t0 < from || t0 + kHalfTokens - 1 > to) {
            // a bit for each token that is seen
            const int32_t last = min(max(top - t0, -1), kHalfTokens - 1);
            const int32_t first = max(bottom - t0, 0);
            const uint64_t seen = last < first ? 0ull : (~0ull >> (63 - last)) & (~0ull << first);
            const uint32_t lo = (uint32_t)seen, hi = (uint32_t)(seen >> 32);
#pragma unroll
            for (int e = 0; e < kHalfTokens; ++e)
              if (!((e < 32 ? lo : hi) & (1u << (e & 31)))) a[e] = 0xff800000u;  // -inf
            // a scale that is no number is not theirs (where they see a token, it is)
#pragma unroll
            for (int g = 0; g < kHalfGroups; ++g)
              if (!((g < 2 ? lo : hi) & (0xffffu << (g & 1) * 16))) {
                by[g] = 1.0f;
                hidden |= 1u << g;
              }
          }
          // ---- the maxima of s and of s + lv
          float b[kHalfGroups];
#pragma unroll
          for (int g = 0; g < kHalfGroups; ++g) b[g] = -INFINITY;
#pragma unroll
          for (int e = 0; e < 16; e += 2)
#pragma unroll
            for (int g = 0; g < kHalfGroups; ++g)
              b[g] = fmaxf(b[g], fmaxf(__uint_as_float(a[g * 16 + e]),
                                       __uint_as_float(a[g * 16 + e + 1])));
          float most = -INFINITY, most_s = -INFINITY;
#pragma unroll
          for (int g = 0; g < kHalfGroups; ++g) {
            const float s = b[g] * by[g];
            most_s = fmaxf(most_s, s);
            most = fmaxf(most, s + lv[g]);
          }
          if (__any_sync(0xffffffffu, most > m + kTilesLag || most_s > ms + kTilesLag)) {
            const float now_s = fmaxf(ms, most_s), now = fmaxf(m, most);
            const float f = m == -INFINITY ? 0.0f : fast_exp2(m - now);
            if (ms != -INFINITY) sum *= fast_exp2(ms - now_s);
            ms = now_s;
            m = now;
            if (u > 0 || half > 0) {                  // once the last half's product is done
              if (!(ok = half ? wait(&sh.o_full[x][0], ns) : wait(&sh.o_full[x][1], ns - 1))) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D / 16; ++c) {
                uint32_t o[16];
                tmem_ld_32x32b_x16(t_o + c * 16, o);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tmem_st_32x32b_x16(t_o + c * 16, o);
              }
            }
          }
          // ---- the weights
          const float shift = ms == -INFINITY ? 0.0f : kTilesShift - ms;
          const float root = m == -INFINITY ? 1.0f : fast_exp2(0.5f * (ms - m));
          const uint64_t shift2 = pack_f32x2(shift, shift);
          uint64_t part[2] = {0, 0};
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t w[16];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int g = c * 2 + y;
              // (a group whose tokens have no weight may have a factor out of range)
              float f = scales[g].z * root * root;
              f = hidden & (1u << g) ? 0.0f : f > kMostFactor ? kMostFactor : f;
              const uint64_t by2 = pack_f32x2(by[g], by[g]), f2 = pack_f32x2(f, f);
#pragma unroll
              for (int e = 0; e < 16; e += 2) {
                const int k = g * 16 + e;
                float z0, z1;
                unpack_f32x2(fma_f32x2(pack_b32x2(a[k], a[k + 1]), by2, shift2), z0, z1);
                const uint64_t z = pack_f32x2(fast_exp2(z0), fast_exp2(z1));
                part[y] = add_f32x2(part[y], z);
                unpack_f32x2(mul_f32x2(z, f2), z0, z1);
                w[y * 8 + e / 2] = half2_of(z0, z1);
              }
            }
            tmem_st_32x32b_x16(t_s + half * 32 + c * 16, w);
          }
          float p0, p1;
          unpack_f32x2(add_f32x2(part[0], part[1]), p0, p1);
          sum += p0 + p1;
          tmem_st_wait();
          tc_fence_before();
          mbar_arrive(&sh.p_full[x][half]);  // (after the second: the scales' place may be written)
        }
        if (!ok) break;
      }
      if (!ok) break;
    }
    cp_async_wait_all();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, 512);
  if (tid == 0 && sh.abort) set_error(p.err, kErrTimeout);
  if (bad) set_error(p.err, bad);
}

template <int D, int FMT>
hs_status launch(const AttendParams& p, cudaStream_t stream) {
  constexpr int smem = TilesLayout<D>::kSmem;
  static std::atomic<uint64_t> configured{0};
  const hs_status st = once_per_device(configured, [] {
    return cuda_fail(cudaFuncSetAttribute(kv_attend_tiles_kernel<D, FMT>,
                                          cudaFuncAttributeMaxDynamicSharedMemorySize, smem),
                     "kv_attend_tiles shared memory");
  });
  if (st != HS_OK) return st;
  // At most an item for every pair of tiles that the batch's rows could fill, in parts.
  const int64_t rows = (int64_t)p.n_tokens * p.G;
  int64_t items = (rows / kPairRows + p.n_req) * p.H * kMostParts;
  if (items > num_sms()) items = num_sms();
  launch_pdl(kv_attend_tiles_kernel<D, FMT>, dim3((unsigned)items), dim3(kTilesThreads), smem,
             stream, p);
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "kv_attend_tiles launch");
}

}  // namespace

// A CTA has a part of an item, where items have parts.
size_t tiles_partial_bytes(int32_t dim) {
  return (size_t)((int64_t)num_sms() * kSoftWarps * 4 *
                  (dim == 64 ? part_floats<64>() : part_floats<128>()));
}

hs_status launch_kv_attend_tiles(const AttendParams& p, int32_t dim, int32_t format,
                                 cudaStream_t stream) {
  if (dim == 64)
    return format == HS_KV_E4M3 ? launch<64, HS_KV_E4M3>(p, stream)
                                : launch<64, HS_KV_INT8>(p, stream);
  return format == HS_KV_E4M3 ? launch<128, HS_KV_E4M3>(p, stream)
                              : launch<128, HS_KV_INT8>(p, stream);
}

}  // namespace hs
