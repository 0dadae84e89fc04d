// Attention of few query rows over the paged 8-bit cache (hs_kv_attend): single tokens, drafts,
// and every other length by groups of rows.
//
// For a request with L tokens in the cache and n queries, query i sits at position L - n + i, and
//   s_ij = scale * q_i . k_j,  o_i = sum_j exp(s_ij - lse_i) v_j,  lse_i = log sum_j exp(s_ij)
// over the keys j < L that it sees.  The keys and values of a kv head are shared by the G query
// heads of its group, so the rows of a tile are (query, head of the group): 8 * NT of them.
//
// Reading the codes once is all the work there is (2 * dim bytes a token against 2 * G flops a
// byte), so the kernel is built around keeping loads in flight:
//  - The work is cut into units of a few hundred tokens of one (request, kv head, group of rows),
//    laid end to end, and every CTA (one an SM) takes an equal share of the list, whatever the
//    lengths are.  Where a
//    (request, head, group) is cut between CTAs, each leaves its partial result in the workspace
//    and the one that comes last merges them in their order: no second launch, and a result that
//    does not depend on which was last.
//  - A warp takes 32 of a unit's tokens through a ring of its own in shared memory (cp.async,
//    codes and scales, tokens past the end and before all windows as zeros, so what stale slots hold
//    is never read) and keeps its own running maxima and sum: no barrier until a (request, head, group)
//    ends.
//  - Products are on mma.sync m16n8k16 with tokens as M and rows as N: a decoding step has 1 to 16
//    rows, which would fill an eighth of a tcgen05 tile's 128, and codes go straight from shared
//    memory to registers as half2 (exact for e4m3 and int8).
// Measured: 256 requests of 1 to 8192 tokens, 32 / 8 heads of 128, 2.1 GB in 338 to 345 us (0.92 of
// the copy rate); 8 of 100 to 1500 in 12.3 us, which are launch and round trips; one of 32,771 in 21.9
// (67 MB, of them what L2 still has).
// Arithmetic: q as half after division by a power of two of its row (exact but below 2^-24 of the
// row's largest), products and sums in fp32.  A row keeps two running maxima (both may lag by 8): mx
// of the scores s and mo of s + log2 vs, with vs the values' scale of a token's block.  The weights'
// sum is of z = 2^(s - mx + 7), the output's weights are w = z * vs * 2^(mx - mo) as half (w <= 2^15;
// what is under 2^-32 of a row's largest is dropped from o, not from lse), and o * 2^(mo - mx) / sum is
// the output.  So a block counts by what its values weigh in that row, not by its scale: one that a
// row does not see, or hardly, takes no bits from the others.
#include <algorithm>

#include "kv_cache.cuh"
#include "kv_attend.cuh"

namespace hs {

hs_status launch_kv_attend_tiles(const AttendParams&, int32_t, int32_t, cudaStream_t);
size_t tiles_partial_bytes(int32_t dim);

namespace {

constexpr int kWarpTokens = 32;                          // of a unit, for each warp
constexpr int kFewRows = 32;                             // of a request: see few_rows
constexpr int kAttStages = 2;
// Codes that the GPU reads in about the time in which a CTA ends one (request, head, group) and
// begins another, 4 us: what equal shares may save by cutting into two of them.
constexpr int kSpareBytes = 25000000;
constexpr float kLag = 8.0f;                             // of the running maximum, in powers of two
constexpr float kShift = 7.0f;
constexpr float kLeastScale = 1.17549435e-38f;           // 2^-126
constexpr float kNone = -3.0e38f;                        // a maximum of nothing, and yet a number
constexpr float kMostFactor = 8.5070592e37f;             // 2^126

// Warps of a CTA, and CTAs of an SM.  Small CTAs side by side go on loading while one of them ends
// a (request, head, group), a single large one leaves few parts of a long one to merge.  8 of 16,000
// tokens take 17.5 us with large CTAs and 21.8 with small ones, 19 of 4000 14.4 and 15.7, 8 of 500 10.4
// and 9.9; 32 of 4000 16.0 and 16.6, of 500 10.7 and 10.3; 64 requests of 2000, 8 heads each, 59 and 52.
template <int D, int NT>
constexpr int few_warps() { return D == 256 ? 7 - NT : 4; }
template <int D, int NT>
constexpr int many_warps() { return D == 256 ? 7 - NT : NT == 1 || (D == 64 && NT == 2) ? 12 : 8; }
template <int D, int NT, int WARPS>
constexpr int attend_ctas() {
  return WARPS > 4 ? 1 : D == 64 ? (NT == 1 ? 4 : NT == 2 ? 3 : 2) : 4 - NT;
}

template <int D>
constexpr int stage_bytes() { return 2 * kWarpTokens * D + 128; }  // K, V, two scales of each

// Where 16-byte chunk c of token row r of a tile lies, so that both ways of reading it (8 tokens
// by 2 chunks, 4 even tokens by 2 chunks) touch every bank once.
template <int D>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
  if constexpr (D == 64)
    return (uint32_t)((r >> 1) * 128 + (((r ^ (r >> 2)) & 1) << 6) + ((c ^ (r & 2)) << 4));
  else
    return (uint32_t)(r * D + (c & ~7) * 16 + (((c ^ r) & 7) << 4));
}

__device__ __forceinline__ void cp_async4_zfill(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src),
               "r"(in ? 4 : 0)
               : "memory");
}

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                          uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}

// A place in the list of units: a (request, kv head, group of rows) and one of its tiles.
struct Place {
  int32_t r, h, group, groups;
  int32_t tile, tile0, tile_end;   // tiles of a CTA's tokens
  int32_t n, q0, len;
};

// The instruction cache is small beside this kernel, and what runs once a request or once a launch
// would push out what runs for every tile: such code stands out of line, or once in a loop.
__device__ __noinline__ int64_t quotient_64(int64_t a, int64_t b) { return a / b; }
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {  // of numbers >= 0
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : quotient_64(a, b);
}

// What a request with n queries over len tokens asks for, in groups of ROWS rows and tiles of TOKENS
// tokens; groups = 0 if nothing, or if it is another kernel's.
struct Request {
  int32_t n, q0, len, groups, tile0, tiles;
  int32_t bad;
};

template <int ROWS, int TOKENS>
__device__ __forceinline__ void divide(const AttendParams& p, Request& q) {
  q.groups = q.tile0 = q.tiles = 0;
  if (q.n == 0 || q.n * p.G > p.rows_most) return;
  q.groups = (q.n * p.G + ROWS - 1) / ROWS;
  q.tile0 = attend_first(p, q.n, q.len) / TOKENS;
  q.tiles = max((q.len + TOKENS - 1) / TOKENS - q.tile0, 1);  // an empty one too
}

template <int ROWS, int TOKENS>
__device__ __noinline__ Request request(const AttendParams& p, int32_t r) {
  Request q{};
  unsigned bad = 0;
  if (!attend_request(p, r, q.n, q.q0, q.len, &bad)) q.n = 0;
  q.bad = (int32_t)bad;
  divide<ROWS, TOKENS>(p, q);
  return q;
}

template <int D, int NT, int WARPS, int FMT>
__global__ void __launch_bounds__(WARPS * 32, attend_ctas<D, NT, WARPS>())
    kv_attend_kernel(const AttendParams p) {
  constexpr int THREADS = WARPS * 32;
  constexpr int TOKENS = WARPS * kWarpTokens;    // of a unit
  constexpr int ROWS = 8 * NT;
  constexpr int HALVES = D == 64 ? 1 : D / 128;  // 128-byte pieces of a row (D = 64: one of 64)
  constexpr int KS = D == 64 ? 4 : 8;            // k16 steps, and m16 tiles of dim, of a piece
  constexpr int NO = HALVES * KS * NT * 4;       // output registers of a thread
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int32_t last_s;
  __shared__ float mx_s[WARPS][ROWS], mo_s[WARPS][ROWS];

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, c = lane & 3;
  uint8_t* ring = smem + warp * (kAttStages * stage_bytes<D>());
  float* merge = reinterpret_cast<float*>(smem + WARPS * kAttStages * stage_bytes<D>());
  const uint32_t ring_u = smem_u32(ring);

  // Beside the kernel of the requests with many rows nothing is waited for: that one has seen to it
  // that what came before is done, and shares no output or workspace with this one.
  if (!p.apart) pdl_wait();
  pdl_trigger();
  const int32_t R = p.n_req_dev ? max(0, min(__ldg(p.n_req_dev), p.n_req)) : p.n_req;

  // ---- how many units there are, and which are this CTA's: each warp for itself, so that no
  // barrier stands before the first loads
  int32_t bad = 0;
  const auto units_of = [&](const Request& q) { return (int64_t)q.groups * q.tiles * p.H; };
  // Of lanes' counts x: up to and with each lane, and all
  const auto scan = [&](int64_t x, int64_t& incl) {
    incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    return __shfl_sync(0xffffffffu, incl, 31);
  };
  constexpr int CHUNKS = 4;
  const bool few = R <= 32 * CHUNKS;
  int64_t n[CHUNKS] = {}, incl[CHUNKS] = {}, all[CHUNKS] = {};
  const int32_t per = (R + 31) / 32;
  Request q[CHUNKS];
  if (few) {                                              // a lane's requests are 32 apart
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      unsigned b = 0;
      q[k] = Request{};
      if (k * 32 + lane < R && !attend_request(p, k * 32 + lane, q[k].n, q[k].q0, q[k].len, &b))
        q[k].n = 0;
      bad |= (int32_t)b;
    }
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      divide<ROWS, TOKENS>(p, q[k]);
      n[k] = units_of(q[k]);
      if (k * 32 < R) all[k] = scan(n[k], incl[k]);
    }
  } else {                                                // they follow each other
#pragma unroll 1
    for (int32_t r = lane * per; r < min((lane + 1) * per, R); ++r) {
      const Request q = request<ROWS, TOKENS>(p, r);
      bad |= q.bad;
      n[0] += units_of(q);
    }
    all[0] = scan(n[0], incl[0]);
  }
  int64_t U = all[0] + all[1] + all[2] + all[3];
  // Where no CTA need have units of two (request, head, group)s, each takes up to `piece` of one, if
  // that is not many more than an equal share: 48 requests of 5 queries, 24 / 4 heads of 64, 43.0 ->
  // 31.4 us; 16 of 4000 tokens, 4 / 1 heads of 128, 17.6 -> 14.3.
  int32_t piece = 0;
  if (few && U > gridDim.x) {
    const auto pieces = [&](int32_t each) {               // of so many units
      int32_t x = 0;
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k)
        if (n[k] > 0) x += q[k].groups * p.H * ((q[k].tiles + each - 1) / each);
      return __reduce_add_sync(0xffffffffu, x);
    };
    if (pieces(1 << 30) <= (int32_t)gridDim.x) {          // (as many as there are of them)
      const int32_t least = (int32_t)quotient(U + gridDim.x - 1, gridDim.x);
      const int32_t most = least + kSpareBytes / ((int32_t)gridDim.x * TOKENS * 2 * D);
#pragma unroll 1
      for (int32_t each = least; each <= most && !piece; ++each)
        if (pieces(each) <= (int32_t)gridDim.x) piece = each;
    }
    if (piece) {                                          // the list with room up to whole pieces
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        if (n[k] > 0) n[k] = (int64_t)q[k].groups * p.H * ((q[k].tiles + piece - 1) / piece) * piece;
        if (k * 32 < R) all[k] = scan(n[k], incl[k]);
      }
      U = all[0] + all[1] + all[2] + all[3];
    }
  }
  if (bad && blockIdx.x == 0) set_error(p.err, (unsigned)bad);
  if (blockIdx.x >= U || (piece && (int64_t)blockIdx.x * piece >= U)) {
    if (p.apart) pdl_wait();
    return;
  }
  const int64_t E = min((int64_t)gridDim.x, U);           // CTAs with work: share units each, and
  const int64_t share = piece ? piece : quotient(U, E);   // the first `longer` one more
  const int64_t longer = piece ? 0 : U - share * E;
  const auto begins = [&](int64_t cta) { return cta * share + min(cta, longer); };
  const auto cta_of = [&](int64_t u) {
    const int64_t cut = longer * (share + 1);
    return (int32_t)(u < cut ? quotient(u, share + 1) : longer + quotient(u - cut, share));
  };
  const int64_t u_begin = begins(blockIdx.x);
  int64_t units = begins(blockIdx.x + 1) - u_begin;
  int64_t skip = u_begin;                                 // units before its first in start_r
  int32_t start_r = 0;
  Request start{};
  if (few) {
    bool found = false;
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      if (!found && skip < all[k]) {
        const int holder = __ffs(__ballot_sync(0xffffffffu, skip < incl[k])) - 1;
        skip -= __shfl_sync(0xffffffffu, incl[k] - n[k], holder);
        start_r = k * 32 + holder;
        start.n = __shfl_sync(0xffffffffu, q[k].n, holder);
        start.q0 = __shfl_sync(0xffffffffu, q[k].q0, holder);
        start.len = __shfl_sync(0xffffffffu, q[k].len, holder);
        found = true;
      }
      if (!found) skip -= all[k];
    }
    divide<ROWS, TOKENS>(p, start);
  } else {
    int holder = __ffs(__ballot_sync(0xffffffffu, skip < incl[0])) - 1;
    skip -= __shfl_sync(0xffffffffu, incl[0] - n[0], holder);
    start_r = holder * per;
    const int32_t end = min(start_r + per, R);
#pragma unroll 1
    for (int32_t base = start_r;; base += 32) {           // which of that lane's it is
      int64_t one = 0, upto;
      if (base + lane < end) one = units_of(request<ROWS, TOKENS>(p, base + lane));
      const int64_t some = scan(one, upto);
      if (skip < some || base + 32 >= end) {
        const unsigned holds = __ballot_sync(0xffffffffu, skip < upto);
        holder = holds ? __ffs(holds) - 1 : 31;
        skip -= __shfl_sync(0xffffffffu, upto - one, holder);
        start_r = base + holder;
        break;
      }
      skip -= some;
    }
    start = request<ROWS, TOKENS>(p, start_r);
  }

  Place fetch{};                                          // what is loaded next
  const auto enter = [&](int32_t r, const Request& w) {
    fetch.r = r;
    fetch.groups = w.groups;
    fetch.n = w.n;
    fetch.q0 = w.q0;
    fetch.len = w.len;
    fetch.tile0 = fetch.tile = w.tile0;
    fetch.tile_end = w.tile0 + w.tiles;
    fetch.h = fetch.group = 0;
  };
  const auto open = [&](int32_t r) {                      // ... the next request with work
    Request w{0, 0, 0, 1, 0, 1, 0};                       // (of none, should the lengths change)
#pragma unroll 1
    for (; r < R; ++r) {
      const Request x = request<ROWS, TOKENS>(p, r);
      if (x.groups > 0) {
        w = x;
        break;
      }
    }
    enter(r, w);
  };

  // ---- loading: this warp's 32 tokens of a unit, one stage
  const int two = p.bt_log2 == 4;                         // its tokens lie in two blocks
  int32_t id0 = 0, id1 = 0;
  const auto look_up = [&]() {                            // the blocks of `fetch`
    const int32_t t0 = fetch.tile * TOKENS + warp * kWarpTokens;
    const int32_t* row = p.table + (int64_t)fetch.r * p.width + (t0 >> p.bt_log2);
    id0 = t0 < fetch.len ? __ldg(row) : 0;
    id1 = two && t0 + 16 < fetch.len ? __ldg(row + 1) : id0;
  };
  const auto load = [&](int stage) {
    const int32_t t0 = fetch.tile * TOKENS + warp * kWarpTokens;
    int32_t left = fetch.len - t0;                        // tokens that there are
    int32_t from = attend_first(p, fetch.n, fetch.len) - t0;  // rows before it are zeros, too
    const bool ok0 = (uint32_t)id0 < (uint32_t)p.n_blocks, ok1 = (uint32_t)id1 < (uint32_t)p.n_blocks;
    if (!ok0 || !ok1) {                                   // ... and those of an entry that is no block
      if (left > 0) set_error(p.err, kErrInvalidArg);
      left = ok0 ? min(left, 16) : ok1 ? left : 0;
      if (!ok0) from = max(from, 16);
      id0 = ok0 ? id0 : 0;                                // (nothing is copied from there)
      id1 = ok1 ? id1 : 0;
    }
    const uint32_t base = ring_u + stage * stage_bytes<D>();
    if (left > 0) {
      const int64_t in = (int64_t)(t0 & ((1 << p.bt_log2) - 1)) * D;
      const int64_t b0 = ((((int64_t)id0 * p.H + fetch.h) << p.bt_log2) * D) + in;
      const int64_t b1 = two ? (((int64_t)id1 * p.H + fetch.h) << 4) * D - 16 * D : b0;
      // A lane's copies are RPI rows, 512 bytes, apart, from its own place in the first rows on;
      // rows past the end are zeros (their addresses are inside the block all the same).
      constexpr int CH = D / 16, RPI = 32 / CH;           // chunks of a row, rows of a copy
      const int r0 = lane / CH;
      const uint8_t* k0 = p.k + b0 + lane * 16;
      const uint8_t* v0 = p.v + b0 + lane * 16;
      const int64_t other = b1 - b0;                      // of the second 16 tokens
      const uint32_t dst = base + chunk_at<D>(r0, lane % CH);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const bool ok = r0 < left - i * RPI && r0 >= from - i * RPI;
        const int64_t off = i * 512 + (i < CH / 2 ? 0 : other);
        const uint32_t to = (dst + i * 512) ^ (D == 64 ? 0 : ((i * RPI) & 7) << 4);
        cp_async16_zfill(to, k0 + off, ok);
        cp_async16_zfill(to + kWarpTokens * D, v0 + off, ok);
      }
      if (lane < 4) {
        const float* s = lane < 2 ? p.ks : p.vs;
        const bool ok = (lane & 1) * 16 < left && (lane & 1) * 16 + 16 > from;
        const int64_t at = (int64_t)((lane & 1) ? id1 : id0) * p.H + fetch.h;
        cp_async4_zfill(base + 2 * kWarpTokens * D + lane * 4, s + (ok ? at : 0), ok);
      }
    } else {
      for (int at = lane * 16; at < stage_bytes<D>(); at += 512)
        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(base + at), "r"(0)
                     : "memory");
    }
  };

  uint32_t qf[HALVES][KS][NT][2];
  float o[HALVES][KS][NT][4];
  float mx[NT][2], mo[NT][2], sum[NT][2], qs[NT][2];
  int32_t top[NT][2], bottom[NT][2];                      // keys that a row sees: bottom .. top
  // A place's queries as they are stored; a thread has row g of each eight, 4 of dim a k16 step.
  const auto load_queries = [&](const Place& w) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = w.group * ROWS + nt * 8 + g;
      const bool in = row < w.n * p.G;
      const int i = in ? attend_query(p, row) : 0, j = in ? row - i * p.G : 0;
      const uint16_t* src = p.q + (int64_t)(w.q0 + i) * p.q_token +
                            (int64_t)(w.h * p.G + j) * p.q_head + c * (KS * 4);
#pragma unroll
      for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
        for (int k = 0; k < KS; k += 2) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);  // (unaligned rows: a call)
          if (in)
            v = p.q_vec ? __ldg(reinterpret_cast<const uint4*>(src + hf * 128 + k * 4))
                        : attend_raw8(src + hf * 128 + k * 4);
          qf[hf][k][nt][0] = v.x;
          qf[hf][k][nt][1] = v.y;
          qf[hf][k + 1][nt][0] = v.z;
          qf[hf][k + 1][nt][1] = v.w;
        }
    }
  };
  // Where in a tile this thread's keys (row g of each eight) and values (rows 2c, 2c + 1) begin:
  // the order of chunks repeats every eight rows.
  uint32_t k_lane[(KS + 3) / 4], v_lane[2];
#pragma unroll
  for (int k = 0; k < (KS + 3) / 4; ++k) k_lane[k] = chunk_at<D>(g, (KS / 4) * c + k);
#pragma unroll
  for (int x = 0; x < 2; ++x)
    v_lane[x] = D == 64 ? chunk_at<D>(2 * c + x, g >> 1) + (g & 1) * 8 : chunk_at<D>(2 * c + x, g);
  bool fresh = true;
  int32_t seg_tile = 0;                                   // the first tile that this CTA has of it
  Place at{}, next{};                                     // what is computed, what was loaded last

  enter(start_r, start);
  if (skip < fetch.tile_end - fetch.tile0) {              // (of the first head and group, mostly)
    fetch.tile += (int32_t)skip;
  } else {
    int32_t tiles = fetch.tile_end - fetch.tile0;
    if (piece) tiles = (tiles + piece - 1) / piece * piece;
    const int64_t part = quotient(skip, tiles);           // which (head, group)
    fetch.tile += (int32_t)(skip - part * tiles);
    fetch.h = (int32_t)quotient(part, fetch.groups);
    fetch.group = (int32_t)(part - (int64_t)fetch.h * fetch.groups);
  }
  if (piece) units = min(piece, fetch.tile_end - fetch.tile);
  look_up();
#pragma unroll 1
  for (int64_t i = 0; i <= units; ++i) {                  // load unit i, compute unit i - 1
    __syncwarp();
    if (i < units) {
      load((int)(i & 1));
      next = fetch;
      if (i + 1 < units) {                                // the next unit of the list, and its blocks
        if (++fetch.tile == fetch.tile_end) {
          fetch.tile = fetch.tile0;
          if (++fetch.group == fetch.groups) {
            fetch.group = 0;
            if (++fetch.h == p.H) open(fetch.r + 1);
          }
        }
        look_up();
      }
    }
    cp_async_commit();
    bool ends = false;
    if (i > 0) {
      const int stage = (int)((i - 1) & 1);
      if (fresh) {                                          // a (request, head, group) begins
        fresh = false;
        seg_tile = at.tile;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float big = 0.0f;
#pragma unroll
          for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float2 f = attend_unpack2(qf[hf][k][nt][e], p.fp16);
                big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
              }
          big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
          big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
          // a power of two of the row's size, kept where it and its inverse are normal
          const uint32_t ex = min(max(__float_as_uint(big) >> 23, 1u), 253u);
          const float by = __uint_as_float((254u - ex) << 23);
#pragma unroll
          for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float2 f = attend_unpack2(qf[hf][k][nt][e], p.fp16);
                qf[hf][k][nt][e] = pack_half2(f.x * by, f.y * by);
              }
          const float back = __uint_as_float(ex << 23) * p.scale_log2;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            qs[nt][e] = __shfl_sync(0xffffffffu, back, (2 * c + e) * 4);
            mx[nt][e] = -INFINITY;
            mo[nt][e] = kNone;
            sum[nt][e] = 0.0f;
            const int pos = at.len - at.n + attend_query(p, at.group * ROWS + nt * 8 + 2 * c + e);
            top[nt][e] = p.causal ? min(pos, at.len - 1) : at.len - 1;
            bottom[nt][e] = p.window > 0 ? pos - attend_window(p, at.len) + 1 : 0;
          }
        }
#pragma unroll
        for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[hf][k][nt][e] = 0.0f;
      }

      cp_async_wait<1>();
      __syncwarp();
      const uint32_t kb = ring_u + stage * stage_bytes<D>(), vb = kb + kWarpTokens * D;
      float scales[4];
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                   : "=f"(scales[0]), "=f"(scales[1]), "=f"(scales[2]), "=f"(scales[3])
                   : "r"(kb + 2 * kWarpTokens * D)
                   : "memory");
      const int32_t t0 = at.tile * TOKENS + warp * kWarpTokens;
      if (t0 < at.len) {
        // ---- s = q . k: tokens are M, rows are N
        float s[2][NT][4];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[mt][nt][e] = 0.0f;
#pragma unroll
          for (int hf = 0; hf < HALVES; ++hf) {
            uint32_t a[2][KS];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
  #pragma unroll
              for (int k = 0; k < KS; k += 4) {
                const uint4 w = lds128(kb + k_lane[k / 4] + hf * 128 + (mt * 16 + x * 8) * D);
                a[x][k] = w.x;
                a[x][k + 1] = w.y;
                a[x][k + 2] = w.z;
                a[x][k + 3] = w.w;
              }
            }
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              const uint32_t a0 = KvFormat<FMT>::template decode2<0>(a[0][k]);
              const uint32_t a1 = KvFormat<FMT>::template decode2<0>(a[1][k]);
              const uint32_t a2 = KvFormat<FMT>::template decode2<1>(a[0][k]);
              const uint32_t a3 = KvFormat<FMT>::template decode2<1>(a[1][k]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                mma_16816(s[mt][nt], a0, a1, a2, a3, qf[hf][k][nt][0], qf[hf][k][nt][1]);
            }
          }
        }
        // Scales that are no number: a key's makes NaN of the scores, a value's of the outputs, of the
        // rows that see one of its tokens.  (Scales are >= 0.)
        if (!((scales[0] + scales[1]) + (scales[2] + scales[3]) < INFINITY)) {
          const float nan = __int_as_float(0x7fffffff);
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            if (!(scales[mt] < INFINITY)) scales[mt] = nan;
            if (scales[2 + mt] < INFINITY) continue;
            scales[2 + mt] = 0.0f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                if (max(t0 + mt * 16, bottom[nt][e]) > min(t0 + mt * 16 + 15, top[nt][e])) continue;
#pragma unroll
                for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
                  for (int k = 0; k < KS; ++k) o[hf][k][nt][e] = o[hf][k][nt][2 + e] = nan;
              }
          }
        }
        // ---- masks, running maxima
        const bool whole = t0 + kWarpTokens <= (p.causal ? at.len - at.n + 1 : at.len) &&
                           (p.window <= 0 || t0 > at.len - 1 - p.window);
        const float lv[2] = {__log2f(fmaxf(scales[2], kLeastScale)),
                             __log2f(fmaxf(scales[3], kLeastScale))};
        float most[NT][2], most_o[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            most[nt][e] = most_o[nt][e] = -INFINITY;
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
              float m = -INFINITY;
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                float& z = s[mt][nt][2 * x + e];
                z *= scales[mt] * qs[nt][e];
                if (!whole) {
                  const int t = t0 + mt * 16 + x * 8 + g;
                  if (t > top[nt][e] || t < bottom[nt][e]) z = -INFINITY;
                }
                m = fmaxf(m, z);
              }
              most[nt][e] = fmaxf(most[nt][e], m);
              most_o[nt][e] = fmaxf(most_o[nt][e], m + lv[mt]);
            }
          }
        bool grow = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            grow |= most[nt][e] > mx[nt][e] + kLag || most_o[nt][e] > mo[nt][e] + kLag;
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float m = most[nt][e], n = most_o[nt][e];
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) {
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
                n = fmaxf(n, __shfl_xor_sync(0xffffffffu, n, x));
              }
              m = fmaxf(m, mx[nt][e]);
              n = fmaxf(n, mo[nt][e]);
              sum[nt][e] *= m == -INFINITY ? 1.0f : fast_exp2(mx[nt][e] - m);
              const float f = fast_exp2(mo[nt][e] - n);
              mx[nt][e] = m;
              mo[nt][e] = n;
#pragma unroll
              for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                  o[hf][k][nt][e] *= f;
                  o[hf][k][nt][2 + e] *= f;
                }
            }
        }
        // ---- the weights, and o += w . v with dim as M, rows as N, tokens as K
        float root[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            root[nt][e] = fast_exp2(0.5f * (mx[nt][e] - mo[nt][e]));
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          uint32_t pb[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float m = mx[nt][e] == -INFINITY ? 0.0f : mx[nt][e] - kShift;
              // (where no token has weight, it may be out of range)
              float f = scales[2 + mt] * root[nt][e] * root[nt][e];
              f = fminf(f, kMostFactor);
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                float& z = s[mt][nt][2 * x + e];
                z = fast_exp2(z - m);
                sum[nt][e] += z;
                z *= f;
              }
            }
            pb[nt][0] = transpose_8x8(pack_half2(s[mt][nt][0], s[mt][nt][1]));
            pb[nt][1] = transpose_8x8(pack_half2(s[mt][nt][2], s[mt][nt][3]));
          }
#pragma unroll
          for (int hf = 0; hf < HALVES; ++hf) {
            uint32_t w[4][KS / 2];                          // tokens 2c, 2c+1, 2c+8, 2c+9
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const uint32_t at_x = vb + v_lane[x & 1] + hf * 128 + (mt * 16 + (x >> 1) * 8) * D;
              if constexpr (D == 64) {
                const uint2 y = lds64(at_x);
                w[x][0] = y.x;
                w[x][1] = y.y;
              } else {
                const uint4 y = lds128(at_x);
                w[x][0] = y.x;
                w[x][1] = y.y;
                w[x][2] = y.z;
                w[x][3] = y.w;
              }
            }
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              const uint32_t sel = (k & 1) ? 0x7362u : 0x5140u;
              const uint32_t lo = __byte_perm(w[0][k / 2], w[1][k / 2], sel);
              const uint32_t hi = __byte_perm(w[2][k / 2], w[3][k / 2], sel);
              const uint32_t a0 = KvFormat<FMT>::template decode2<0>(lo);
              const uint32_t a1 = KvFormat<FMT>::template decode2<1>(lo);
              const uint32_t a2 = KvFormat<FMT>::template decode2<0>(hi);
              const uint32_t a3 = KvFormat<FMT>::template decode2<1>(hi);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                mma_16816(o[hf][k][nt], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
            }
          }
        }
      }
      ends = at.tile + 1 == at.tile_end || i == units;
    }
    // The next one's queries are on their way while a (request, head, group) ends.
    if ((i == 0 || ends) && i < units) load_queries(next);
    const Place done = at;
    at = next;
    if (!ends) continue;

    // ---- the CTA's part of this (request, head, group) is done: its warps' results together
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1)
          sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], x);
        if (g == 0) {
          mx_s[warp][nt * 8 + 2 * c + e] = mx[nt][e];
          mo_s[warp][nt * 8 + 2 * c + e] = mo[nt][e];
        }
      }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float m = -INFINITY, n = kNone;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          m = fmaxf(m, mx_s[w][nt * 8 + 2 * c + e]);
          n = fmaxf(n, mo_s[w][nt * 8 + 2 * c + e]);
        }
        sum[nt][e] *= mx[nt][e] == -INFINITY ? 0.0f : fast_exp2(mx[nt][e] - m);
        const float f = fast_exp2(mo[nt][e] - n);
        mx[nt][e] = m;                                      // of the CTA from here on
        mo[nt][e] = n;
#pragma unroll
        for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            o[hf][k][nt][e] *= f;
            o[hf][k][nt][2 + e] *= f;
          }
      }
#pragma unroll 1
    for (int live = WARPS; live > 1; live = (live + 1) / 2) {  // the upper half onto the lower
      const int half = (live + 1) / 2;
      if (warp >= half && warp < live) {
        float* d = merge + (warp - half) * (NO + 2 * NT) * 32 + lane;
#pragma unroll
        for (int i = 0; i < NO; ++i) d[i * 32] = (&o[0][0][0][0])[i];
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) d[(NO + i) * 32] = (&sum[0][0])[i];
      }
      __syncthreads();
      if (warp < live - half) {
        const float* d = merge + warp * (NO + 2 * NT) * 32 + lane;
#pragma unroll
        for (int i = 0; i < NO; ++i) (&o[0][0][0][0])[i] += d[i * 32];
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) (&sum[0][0])[i] += d[(NO + i) * 32];
      }
      __syncthreads();
    }
    const bool all_of_it = seg_tile == done.tile0 && done.tile + 1 == done.tile_end;
    // Output of rows by threads that hold values of dim 16 g + 2 k + {0, 1} (D = 64: 8 g + ...)
    const auto write = [&]() {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = done.group * ROWS + nt * 8 + 2 * c + e;
          if (row >= done.n * p.G) continue;
          const int i = attend_query(p, row), j = row - i * p.G;
          const int64_t r = (int64_t)(done.q0 + i) * (p.H * p.G) + done.h * p.G + j;
          const float l = sum[nt][e];
          const bool none = l == 0.0f;
          // 2^(mo - mx) / sum in two factors, which are in range where the output is
          const float back = none ? 0.0f : fast_exp2(0.5f * (mo[nt][e] - mx[nt][e]));
          const float inv = none ? 0.0f : __fdividef(back, l);
#pragma unroll
          for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
            for (int k = 0; k < KS; k += 4) {
              uint32_t w[4];
#pragma unroll
              for (int q = 0; q < 4; ++q)
                w[q] = none ? 0u
                            : attend_pack2(p.fp16, o[hf][k + q][nt][e] * inv * back,
                                           o[hf][k + q][nt][2 + e] * inv * back);
              *reinterpret_cast<uint4*>(p.out + r * D + hf * 128 + g * (2 * KS) + 2 * k) =
                  make_uint4(w[0], w[1], w[2], w[3]);
            }
          if (g == 0 && p.lse)
            p.lse[r] = none ? -INFINITY : (mx[nt][e] - kShift + log2f(l)) * 0.69314718055994531f;
        }
    };
    if (all_of_it) {
      if (warp == 0) write();
    } else {
      // Partial results: the part that begins at this CTA's first unit in its slot 0, one that
      // begins later (and so runs past its last) in slot 1.  A slot is its rows' sums of weights, as
      // log2 of what they are with mx, their mo, and the sums of weighted values [row][dim].
      const int64_t first = u_begin + i - 1 - (done.tile - done.tile0);   // units of the whole
      const int64_t last = first + (done.tile_end - done.tile0) - 1;
      const int32_t c0 = cta_of(first), c1 = cta_of(last);
      constexpr int PS = ROWS * (D + 2);
      const int32_t odd = first > begins(c0) ? 1 : 0;                  // the first part's slot
      const auto slot_of = [&](int32_t k) {                           // of part k
        return p.partial + ((int64_t)(c0 + k) * 2 + (k == 0 ? odd : 0)) * PS;
      };
      if (warp == 0) {
        float* d = slot_of((int32_t)blockIdx.x - c0);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int row = nt * 8 + 2 * c + e;
            if (g == 0) {
              __stcg(d + row, mx[nt][e] + log2f(sum[nt][e]));   // (-inf of none)
              __stcg(d + ROWS + row, mo[nt][e]);
            }
#pragma unroll
            for (int hf = 0; hf < HALVES; ++hf)
#pragma unroll
              for (int k = 0; k < KS; k += 2)
                __stcg(reinterpret_cast<float4*>(d + 2 * ROWS + row * D + hf * 128 +
                                                 g * (2 * KS) + 2 * k),
                       make_float4(o[hf][k][nt][e], o[hf][k][nt][2 + e], o[hf][k + 1][nt][e],
                                   o[hf][k + 1][nt][2 + e]));
          }
        __threadfence();
        __syncwarp();
        if (lane == 0) last_s = atomicAdd(p.counters + c0, 1u) == (unsigned)(c1 - c0);
      }
      __syncthreads();
      if (last_s) {                                       // everyone else has left its part
        __threadfence();
        const int32_t parts = c1 - c0 + 1;
        // A thread has NF times four values, THREADS apart; UN parts of them on their way at once.
        constexpr int NF = (ROWS * D / 4 + THREADS - 1) / THREADS;
        constexpr int UN = NF >= 4 ? 1 : NF >= 2 ? 3 : 9;
        float4 acc[NF];
        float m[NF], mo[NF], l[NF];
#pragma unroll
        for (int i = 0; i < NF; ++i) {
          acc[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          m[i] = -INFINITY;
          mo[i] = kNone;
          l[i] = 0.0f;
        }
        for (int32_t k0 = 0; k0 < parts; k0 += UN) {
          float4 v[NF][UN];
          float pm[NF][UN], po[NF][UN];
#pragma unroll
          for (int y = 0; y < UN; ++y) {
            const bool in = k0 + y < parts;
            const float* d = slot_of(in ? k0 + y : k0);
#pragma unroll
            for (int i = 0; i < NF; ++i) {
              const int f = min(tid + i * THREADS, ROWS * D / 4 - 1), row = f / (D / 4);
              pm[i][y] = in ? __ldcg(d + row) : -INFINITY;
              po[i][y] = in ? __ldcg(d + ROWS + row) : kNone;
              v[i][y] = __ldcg(reinterpret_cast<const float4*>(d + 2 * ROWS) + f);
            }
          }
#pragma unroll
          for (int i = 0; i < NF; ++i) {
            float now = m[i], now_o = mo[i];
#pragma unroll
            for (int y = 0; y < UN; ++y) {
              now = fmaxf(now, pm[i][y]);
              now_o = fmaxf(now_o, po[i][y]);
            }
            const float back = fast_exp2(mo[i] - now_o);
            l[i] *= m[i] == -INFINITY ? 0.0f : fast_exp2(m[i] - now);
            m[i] = now;
            mo[i] = now_o;
            acc[i].x *= back;
            acc[i].y *= back;
            acc[i].z *= back;
            acc[i].w *= back;
#pragma unroll
            for (int y = 0; y < UN; ++y) {
              l[i] += pm[i][y] == -INFINITY ? 0.0f : fast_exp2(pm[i][y] - now);
              const float w = fast_exp2(po[i][y] - now_o);
              acc[i].x = fmaf(w, v[i][y].x, acc[i].x);
              acc[i].y = fmaf(w, v[i][y].y, acc[i].y);
              acc[i].z = fmaf(w, v[i][y].z, acc[i].z);
              acc[i].w = fmaf(w, v[i][y].w, acc[i].w);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < NF; ++i) {
          const int f = tid + i * THREADS, row = f / (D / 4), full = done.group * ROWS + row;
          if (f >= ROWS * D / 4 || full >= done.n * p.G) continue;
          const int a = attend_query(p, full), b = full - a * p.G;
          const int64_t r = (int64_t)(done.q0 + a) * (p.H * p.G) + done.h * p.G + b;
          const bool none = l[i] == 0.0f;
          const float back = none ? 0.0f : fast_exp2(0.5f * (mo[i] - m[i]));
          const float inv = none ? 0.0f : __fdividef(back, l[i]);
          uint2 w = make_uint2(0u, 0u);
          if (!none) {
            w.x = attend_pack2(p.fp16, acc[i].x * inv * back, acc[i].y * inv * back);
            w.y = attend_pack2(p.fp16, acc[i].z * inv * back, acc[i].w * inv * back);
          }
          *reinterpret_cast<uint2*>(p.out + r * D + (f - row * (D / 4)) * 4) = w;
          if (f == row * (D / 4) && p.lse)
            p.lse[r] = none ? -INFINITY : (m[i] - kShift + log2f(l[i])) * 0.69314718055994531f;
        }
        __syncthreads();
        if (tid == 0) p.counters[c0] = 0;                 // as the next call finds it
      }
      __syncthreads();
    }
    fresh = true;
  }
  cp_async_wait_all();
  if (p.apart) pdl_wait();
}

template <int D, int NT, int WARPS>
constexpr size_t attend_smem() {
  constexpr int NO = D / 16 * NT * 4;
  return (size_t)WARPS * kAttStages * stage_bytes<D>() +
         (size_t)(WARPS / 2) * (NO + 2 * NT) * 32 * 4;
}

template <int D, int NT, int WARPS, int FMT>
hs_status launch(const AttendParams& p, cudaStream_t stream) {
  constexpr int smem = (int)attend_smem<D, NT, WARPS>();
  static std::atomic<uint64_t> configured{0};
  const hs_status st = once_per_device(configured, [] {
    return cuda_fail(cudaFuncSetAttribute(kv_attend_kernel<D, NT, WARPS, FMT>,
                                          cudaFuncAttributeMaxDynamicSharedMemorySize, smem),
                     "kv_attend shared memory");
  });
  if (st != HS_OK) return st;
  launch_pdl(kv_attend_kernel<D, NT, WARPS, FMT>,
             dim3((unsigned)(num_sms() * attend_ctas<D, NT, WARPS>())), dim3(WARPS * 32), smem,
             stream, p);
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "kv_attend launch");
}

template <int D, int NT, int FMT>
hs_status launch_warps(const AttendParams& p, int64_t rows, cudaStream_t stream) {
  // (request, head, group)s, at most
  const int64_t whole = (int64_t)p.n_req * p.H * ((rows + 8 * NT - 1) / (8 * NT));
  return whole * 8 <= num_sms() ? launch<D, NT, many_warps<D, NT>(), FMT>(p, stream)
                                : launch<D, NT, few_warps<D, NT>(), FMT>(p, stream);
}

template <int D, int FMT>
hs_status launch_rows(const AttendParams& p, int64_t rows, cudaStream_t stream) {
  if (rows <= 8) return launch_warps<D, 1, FMT>(p, rows, stream);
  // With dim = 64 there are registers for 32 rows: the codes are read and decoded once for them.
  if constexpr (D == 64)
    if (rows > 16) return launch_warps<D, 4, FMT>(p, rows, stream);
  return launch_warps<D, 2, FMT>(p, rows, stream);
}

template <int FMT>
hs_status launch_dim(const AttendParams& p, int32_t dim, int64_t rows, cudaStream_t stream) {
  return dim == 64    ? launch_rows<64, FMT>(p, rows, stream)
         : dim == 128 ? launch_rows<128, FMT>(p, rows, stream)
                      : launch_rows<256, FMT>(p, rows, stream);
}

}  // namespace

// Rows of a request up to which this kernel takes it, where kv_attend_tiles.cu could.  There up to
// 256 rows cost what one does, here every 16 read the codes again: 64 requests of 2000 tokens, 8
// heads of 128, take 126 us here and 164 there with 32 rows, 232 and 165 with 64.  But there eight
// CTAs share an item at most, here as many as there are: one request of 8192 tokens, one head and
// 512 rows takes 28 us here and 41 there, one of 2000 tokens, 8 heads and 64 rows 18 and 26.  The two
// are level at about one (request, head, 16 rows) for two SMs.
static int32_t few_rows(const AttendParams& p) {
  const int64_t heads = (int64_t)p.n_req * p.H;
  return (int32_t)std::max<int64_t>(kFewRows, num_sms() / (2 * heads) * 16);
}

static size_t few_partial_bytes(int32_t dim) {
  const int64_t rows = dim == 64 ? 32 : 16;               // of a tile, at most
  const int64_t ctas = (int64_t)num_sms() * kAttendMaxPerSm;
  return (size_t)(ctas * 2 * rows * (dim + 2) * 4);
}

// `rows`: of a request, at most
size_t attend_workspace(int32_t dim, int64_t rows) {
  return attend_counter_bytes() + few_partial_bytes(dim) +
         (dim <= 128 && rows > kFewRows ? tiles_partial_bytes(dim) : 0);
}

hs_status launch_kv_attend(AttendParams p, int32_t dim, int32_t format, int64_t rows, void* ws,
                           cudaStream_t stream) {
  p.err = device_error_word();
  if (!p.err) return fail(HS_ERR_CUDA, "could not resolve the device error word");
  p.counters = static_cast<unsigned*>(ws);
  p.queue = p.counters + attend_counters();
  p.tile_counters = p.queue + 2;
  p.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + attend_counter_bytes());
  p.tile_partial = p.partial + few_partial_bytes(dim) / 4;
  p.rows_most = 0x7fffffff;
  const int32_t few = few_rows(p);
  if (dim <= 128 && rows > few) {
    // Requests of many rows by tiles; with lengths of their own there may be others.
    p.rows_most = few;
    if (const hs_status st = launch_kv_attend_tiles(p, dim, format, stream)) return st;
    if (!p.starts) return HS_OK;
    p.apart = 1;
    rows = few;
  }
  return format == HS_KV_E4M3 ? launch_dim<HS_KV_E4M3>(p, dim, rows, stream)
                              : launch_dim<HS_KV_INT8>(p, dim, rows, stream);
}

}  // namespace hs
