// Attention of many query rows over the paged 8-bit cache (hs_kv_attend): prompts, chunks and
// cross attention, on the tensor cores.
//
// The formula is kv_attend.cu's.  A tile is 128 rows (query, head of the group) against 128
// tokens: s = q k^T is one tcgen05.mma per 16 of dim (M = 128, N = 128) into tensor memory, o += p v
// one per 16 tokens (N = dim) with p as its A operand in tensor memory.  4 flops a (row, token, dim)
// and one exponential a (row, token): tensor cores and exponentials bound it together, so a CTA
// keeps two tiles of rows in flight that take turns: while one's scores become weights, the tensor
// cores work for the other.
//
//   warps 0-3, 4-7   a thread a row: scores to weights, the output at the end
//   warps 8-11       queries, and codes from the cache's blocks, decoded to half in shared memory
//                    (swizzled; K and V alike: K is read along dim, V across it)
//   warp 12          one thread issues every product
//
// CTAs are persistent, one an SM.  Work is (request, pair of tiles of rows, kv head) items, the
// later pairs of a request (which see more) first; an item's queries and first tokens are loaded
// while the one before it ends.
//
// Arithmetic: q as half after division by a power of two of its row; codes as half (exact); sums
// in fp32.  A block's scales enter through the exponent: with c the scores' factor and lv = log2 of
// the values' scale, p' = 2^(acc * c + lv - m + 7) with m the running maximum of acc * c + lv
// (it may lag by 8), o = sum p' code, and the weights' sum takes each block's p' / 2^lv.  So value
// scales may be as far apart as they like.
#include "kv_attend.cuh"
#include "kv_cache.cuh"

namespace hs {
namespace {

constexpr int kTileRows = 128;
constexpr int kPairRows = 2 * kTileRows;
constexpr int kTileTokens = 128;
constexpr int kGroups = kTileTokens / 16;      // 16 tokens lie in one block: one scale
constexpr int kSoftWarps = 8;
constexpr int kLoadWarp = 8;                   // the first of four
constexpr int kMmaWarp = 12;
constexpr int kTilesThreads = 13 * 32;
constexpr int kLoadThreads = 128;
constexpr int kScaleRing = 4;
constexpr float kTilesLag = 8.0f;
constexpr float kTilesShift = 7.0f;
constexpr float kLeastScale = 1.17549435e-38f;

template <int D>
struct TilesLayout {
  static constexpr int kBlockBytes = 128 * 128;              // 64 of dim, 128 rows
  static constexpr int kTileBytes = D / 64 * kBlockBytes;    // 128 rows or tokens of dim as half
  static constexpr int kQ = 0;                               // two tiles
  static constexpr int kK = 2 * kTileBytes;                  // two stages
  static constexpr int kV = 4 * kTileBytes;                  // two stages
  static constexpr int kEnd = 6 * kTileBytes;
  static constexpr int kSmem = kEnd + 1024;                  // the base is aligned to 1024
};

struct Item {
  int32_t r, h, rows0, n, q0, len;
  int32_t tile0, tiles, rows;        // tiles of tokens; rows of the request
  int32_t more;                      // 0: no further item
};

struct TilesShared {
  uint64_t q_full, q_empty;
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t s_full[2], p_full[2], o_full[2];
  uint64_t drained;
  Item item;
  float q_scale[kPairRows];
  float4 scales[kScaleRing][kGroups];   // of 16 tokens: keys', log2 of values', 1 / values'
  uint32_t tmem;
  int abort;
  int32_t sums[kTilesThreads / 32];
  int32_t before[kTilesThreads + 1];    // items before each thread's requests
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

__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
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
    mbar_init(&sh.q_full, kLoadThreads);
    mbar_init(&sh.q_empty, kSoftWarps + 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.k_full[i], kLoadThreads);
      mbar_init(&sh.k_empty[i], 1);
      mbar_init(&sh.v_full[i], kLoadThreads);
      mbar_init(&sh.v_empty[i], 1);
      mbar_init(&sh.s_full[i], 2);
      mbar_init(&sh.p_full[i], kTileRows);
      mbar_init(&sh.o_full[i], 1);
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
    Item it;
    for (int32_t r = ra; r < rb; ++r) mine += request_pairs(p, r, it, &bad);
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
  const int32_t total = sh.before[kTilesThreads];
  const uint32_t tmem = sh.tmem;
  volatile int* abort = &sh.abort;
  const auto wait_one = [&](uint64_t* bar, uint32_t phase) {
    return mbar_wait(bar, phase & 1u, abort);
  };
  const auto wait = [&](uint64_t* bar, uint32_t phase) {  // a warp goes on, or gives up, as one
    return __all_sync(0xffffffffu, mbar_wait(bar, phase & 1u, abort)) != 0;
  };

  if (warp >= kLoadWarp && warp < kMmaWarp) {
    // ================================ queries, keys and values
    const int lw = warp - kLoadWarp, lt = tid - kLoadWarp * 32;
    uint32_t items = 0, tiles = 0;                  // done so far, of this CTA
    bool ok = true;
    for (int32_t at = blockIdx.x;; at += gridDim.x, ++items) {
      Item it{};
      it.more = at < total;
      if (it.more) {
        int lo = 0, hi = kTilesThreads;             // the last thread with before <= at
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (sh.before[mid] <= at) lo = mid; else hi = mid;
        }
        int32_t x = at - sh.before[lo], pairs = 0;
        int32_t r = lo * per;
        for (;; ++r) {
          pairs = request_pairs(p, r, it, &bad);
          if (x < pairs * p.H || r + 1 >= min((lo + 1) * per, R)) break;
          x -= pairs * p.H;
        }
        it.r = r;
        it.h = x % p.H;
        it.rows0 = max(pairs - 1 - x / p.H, 0) * kPairRows;
        const int32_t i0 = it.rows0 / p.G, i1 = min(it.n - 1, (it.rows0 + kPairRows - 1) / p.G);
        const int32_t see = p.causal ? min(it.len, it.len - it.n + i1 + 1) : it.len;
        const int32_t from = p.window > 0 ? max(0, it.len - it.n + i0 - p.window + 1) : 0;
        it.tile0 = from / kTileTokens;
        it.tiles = max(0, (see + kTileTokens - 1) / kTileTokens - it.tile0);
      }
      if (items > 0 && !(ok = wait(&sh.q_empty, items - 1))) break;
      if (lt == 0) sh.item = it;
      if (!it.more) {
        mbar_arrive(&sh.q_full);
        break;
      }

      // the tokens' codes are on their way while the queries are laid out
      constexpr int CH = D / 64;                    // loads of 64 bytes of a token's codes
      const int row8 = lane & 7, chunk = lane >> 3;
      uint4 kr[4][CH], vr[4][CH];
      float4 sc = make_float4(0.f, 0.f, 0.f, 0.f);
      int32_t ids[2];
      const auto look_up = [&](int32_t t) {         // the blocks of this warp's 32 tokens
        const int32_t t0 = (it.tile0 + t) * kTileTokens + lw * 32;
        const int32_t* row = p.table + (int64_t)it.r * p.width;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int32_t tok = t0 + i * 16;
          ids[i] = tok < it.len ? __ldg(row + (tok >> p.bt_log2)) : -1;
          if (tok < it.len && (uint32_t)ids[i] >= (uint32_t)p.n_blocks) {
            bad = kErrInvalidArg;
            ids[i] = -1;
          }
        }
      };
      const auto fetch = [&](const uint8_t* codes, int32_t t, uint4 (&to)[4][CH]) {
        const int32_t t0 = (it.tile0 + t) * kTileTokens + lw * 32;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int32_t tok = t0 + g * 8 + row8, id = ids[g >> 1];
          const bool in = tok < it.len && id >= 0;
          const uint8_t* src =
              codes + (((((int64_t)(in ? id : 0) * p.H + it.h) << p.bt_log2) +
                        (tok & ((1 << p.bt_log2) - 1))) * D) + chunk * 16;
#pragma unroll
          for (int c = 0; c < CH; ++c)
            to[g][c] = in ? __ldg(reinterpret_cast<const uint4*>(src + c * 64))
                          : make_uint4(0u, 0u, 0u, 0u);
        }
      };
      const auto fetch_scale = [&]() {
        if (lane < 2) {
          const int32_t id = lane ? ids[1] : ids[0];
          const float a = id >= 0 ? __ldg(p.ks + (int64_t)id * p.H + it.h) : 0.0f;
          const float b = id >= 0 ? __ldg(p.vs + (int64_t)id * p.H + it.h) : 0.0f;
          const float v = b < kLeastScale ? kLeastScale : b;      // (a NaN stays one)
          sc = make_float4(a < kLeastScale ? kLeastScale : a, log2f(v), __fdividef(1.0f, v), 0.f);
        }
      };
      const auto put = [&](uint32_t to, const uint4 (&from)[4][CH]) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int row = lw * 32 + g * 8 + row8;
#pragma unroll
          for (int c = 0; c < CH; ++c) {
            const uint32_t w[4] = {from[g][c].x, from[g][c].y, from[g][c].z, from[g][c].w};
            uint32_t h[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              h[2 * i] = KvFormat<FMT>::template decode2<0>(w[i]);
              h[2 * i + 1] = KvFormat<FMT>::template decode2<1>(w[i]);
            }
            const uint32_t line = to + c * L::kBlockBytes + row * 128;
            sts128(line + (((2 * chunk) ^ row8) << 4), h[0], h[1], h[2], h[3]);
            sts128(line + (((2 * chunk + 1) ^ row8) << 4), h[4], h[5], h[6], h[7]);
          }
        }
      };
      if (it.tiles > 0) {
        look_up(0);
        fetch(p.k, 0, kr);
        fetch(p.v, 0, vr);
        fetch_scale();
      }
      // queries: D / 8 lanes a row, 8 values each
      {
        constexpr int LR = D / 8, RS = 32 / LR;     // lanes of a row, rows of a step
        constexpr int UN = 4;
        const int32_t rows = min(it.rows - it.rows0, kPairRows);
        for (int s = lw * RS; s < kPairRows; s += 4 * RS * UN) {
          float f[UN][8];
#pragma unroll
          for (int u = 0; u < UN; ++u) {
            const int row = s + u * 4 * RS + lane / LR;
#pragma unroll
            for (int e = 0; e < 8; ++e) f[u][e] = 0.0f;
            if (row < rows) {
              const int32_t full = it.rows0 + row, i = full / p.G, j = full - i * p.G;
              attend_load8(p.q + (int64_t)(it.q0 + i) * p.q_token +
                               (int64_t)(it.h * p.G + j) * p.q_head + (lane % LR) * 8,
                           p.q_vec, p.fp16, f[u]);
            }
          }
#pragma unroll
          for (int u = 0; u < UN; ++u) {
            const int row = s + u * 4 * RS + lane / LR;
            float big = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) big = fmaxf(big, fabsf(f[u][e]));
#pragma unroll
            for (int o = 1; o < LR; o <<= 1)
              big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
            const uint32_t e = min(max(__float_as_uint(big) >> 23, 1u), 253u);
            const float by = __uint_as_float((254u - e) << 23);
            const int ch = lane % LR;               // 16-byte chunk of the row
            const uint32_t line = base + L::kQ + (row >> 7) * L::kTileBytes +
                                  (ch >> 3) * L::kBlockBytes + (row & 127) * 128;
            sts128(line + (((ch ^ row) & 7) << 4), half2_of(f[u][0] * by, f[u][1] * by),
                   half2_of(f[u][2] * by, f[u][3] * by), half2_of(f[u][4] * by, f[u][5] * by),
                   half2_of(f[u][6] * by, f[u][7] * by));
            if (ch == 0) sh.q_scale[row] = __uint_as_float(e << 23) * p.scale_log2;
          }
        }
      }
      fence_async_shared();
      mbar_arrive(&sh.q_full);

      for (int32_t t = 0; t < it.tiles && ok; ++t, ++tiles) {
        const uint32_t st = tiles & 1, use = tiles >> 1;
        if (tiles >= 2 && !(ok = wait(&sh.k_empty[st], use - 1))) break;
        if (lane < 2) sh.scales[tiles & (kScaleRing - 1)][lw * 2 + lane] = sc;
        put(base + L::kK + st * L::kTileBytes, kr);
        fence_async_shared();
        mbar_arrive(&sh.k_full[st]);
        if (t + 1 < it.tiles) {
          look_up(t + 1);
          fetch(p.k, t + 1, kr);
          fetch_scale();
        }
        if (tiles >= 2 && !(ok = wait(&sh.v_empty[st], use - 1))) break;
        put(base + L::kV + st * L::kTileBytes, vr);
        fence_async_shared();
        mbar_arrive(&sh.v_full[st]);
        if (t + 1 < it.tiles) fetch(p.v, t + 1, vr);
      }
      if (!ok) break;
    }
  } else if (warp == kMmaWarp) {
    // ================================ products
    if (lane == 0) {
      constexpr uint32_t id_qk = idesc_f16(kTileRows, kTileTokens, false);
      constexpr uint32_t id_pv = idesc_f16(kTileRows, D, true);
      uint32_t tiles = 0, np[2] = {0, 0};
      const auto qk = [&](int x, uint32_t st) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = (k >> 2) * L::kBlockBytes + (k & 3) * 32;
          umma_ss(tmem + x * kTileTokens, smem_desc_k_sw128(base + L::kQ + x * L::kTileBytes + off),
                  smem_desc_k_sw128(base + L::kK + st * L::kTileBytes + off), id_qk, k > 0);
        }
      };
      const auto pv = [&](int x, uint32_t st, bool add) {
#pragma unroll
        for (int k = 0; k < kTileTokens / 16; ++k)
          umma_ts(tmem + 2 * kTileTokens + x * D, tmem + x * kTileTokens + k * 8,
                  smem_desc_mn_sw128(base + L::kV + st * L::kTileBytes + k * 2048, L::kBlockBytes),
                  id_pv, add || k > 0);
      };
      // The arrival of this thread's own passes on what it has seen: the block scales.
      const auto scored = [&](int x) {
        umma_commit(&sh.s_full[x]);
        mbar_arrive(&sh.s_full[x]);
      };
      bool ok = true;
      for (uint32_t items = 0; ok; ++items) {
        if (!(ok = wait_one(&sh.q_full, items))) break;
        tc_fence_after();
        const Item it = sh.item;
        if (!it.more) break;
        const bool two = it.rows - it.rows0 > kTileRows;
        if (it.tiles == 0) {
          mbar_arrive(&sh.q_empty);
          continue;
        }
        for (int32_t t = 0; t < it.tiles; ++t, ++tiles) {
          const uint32_t st = tiles & 1, use = tiles >> 1;
          if (!(ok = wait_one(&sh.k_full[st], use))) break;
          tc_fence_after();
          qk(0, st);
          scored(0);
          if (two) {
            if (t > 0) {
              if (!(ok = wait_one(&sh.p_full[1], np[1]++))) break;
              tc_fence_after();
              pv(1, st ^ 1, t > 1);
              umma_commit(&sh.o_full[1]);
              umma_commit(&sh.v_empty[st ^ 1]);
            }
            qk(1, st);
            scored(1);
          }
          umma_commit(&sh.k_empty[st]);
          if (t + 1 == it.tiles) umma_commit(&sh.q_empty);
          if (!(ok = wait_one(&sh.v_full[st], use))) break;
          if (!(ok = wait_one(&sh.p_full[0], np[0]++))) break;
          tc_fence_after();
          pv(0, st, t > 0);
          umma_commit(&sh.o_full[0]);
          if (!two) umma_commit(&sh.v_empty[st]);
        }
        if (!ok) break;
        if (two) {
          const uint32_t st = (tiles - 1) & 1;
          if (!(ok = wait_one(&sh.p_full[1], np[1]++))) break;
          tc_fence_after();
          pv(1, st, it.tiles > 1);
          umma_commit(&sh.o_full[1]);
          umma_commit(&sh.v_empty[st]);
        }
      }
      umma_commit(&sh.drained);                     // nothing of it runs on when memory is given back
      if (!mbar_wait_limit(&sh.drained, 0, abort, kWaitLimitNs)) {
        const uint64_t t0 = globaltimer_ns();       // someone gave up: wait for what was issued
        while (!mbar_try_wait(smem_u32(&sh.drained), 0) && globaltimer_ns() - t0 < kWaitLimitNs) {
        }
      }
    }
    __syncwarp();
  } else {
    // ================================ scores to weights, and the output
    const int x = warp >> 2;                        // which tile of rows
    const int row = (warp & 3) * 32 + lane;         // of it, and lane of tensor memory
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + x * kTileTokens;
    const uint32_t t_o = tmem + lanes + 2 * kTileTokens + x * D;
    uint32_t tiles = 0, ns = 0;                     // of the CTA; of this group
    bool ok = true;
    for (uint32_t items = 0; ok; ++items) {
      if (!(ok = wait(&sh.q_full, items))) break;
      const Item it = sh.item;
      const float qs = sh.q_scale[x * kTileRows + row];
      __syncwarp();
      if (!it.more) break;
      if (lane == 0) mbar_arrive(&sh.q_empty);
      const int32_t rows0 = it.rows0 + x * kTileRows;
      if (rows0 >= it.rows) {                       // no rows of this item are this group's
        tiles += it.tiles;
        continue;
      }
      const int32_t full = min(rows0 + row, it.rows - 1);
      const int32_t i = full / p.G, j = full - i * p.G;
      const int32_t pos = it.len - it.n + i;
      const int32_t top = p.causal ? min(pos, it.len - 1) : it.len - 1;
      const int32_t bottom = p.window > 0 ? pos - p.window + 1 : 0;
      // tokens that every row of the tile sees: from .. to
      const int32_t pos0 = it.len - it.n + rows0 / p.G;
      const int32_t pos1 = it.len - it.n + min(it.n - 1, (rows0 + kTileRows - 1) / p.G);
      const int32_t to = p.causal ? min(pos0, it.len - 1) : it.len - 1;
      const int32_t from = p.window > 0 ? pos1 - p.window + 1 : 0;

      float m = -INFINITY, sum = 0.0f;
      for (int32_t t = 0; t < it.tiles; ++t, ++tiles, ++ns) {
        if (!(ok = wait(&sh.s_full[x], ns))) break;
        tc_fence_after();
        const float4* scales = sh.scales[tiles & (kScaleRing - 1)];
        const int32_t t0 = (it.tile0 + t) * kTileTokens;
        const bool whole = t0 >= from && t0 + kTileTokens - 1 <= to;
        const int32_t last = top - t0, first = bottom - t0;
        // ---- the maximum of acc * c + lv
        float most = -INFINITY;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t a[32];
          tmem_ld_32x32b_x32(t_s + c * 32, a);
          tmem_ld_wait();
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const float4 sc = scales[c * 2 + g];
            float b = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float z = __uint_as_float(a[g * 16 + e]);
              if (!whole) {
                const int32_t tok = c * 32 + g * 16 + e;
                if (tok > last || tok < first) z = -INFINITY;
              }
              b = fmaxf(b, z);
            }
            most = fmaxf(most, fmaf(b, factor(sc.x, qs), sc.y));
          }
        }
        const bool grow = most > m + kTilesLag;
        if (__any_sync(0xffffffffu, grow)) {
          const float now = fmaxf(m, most);
          const float f = m == -INFINITY ? 0.0f : fast_exp2(m - now);
          m = now;
          sum *= f;
          if (t > 0) {
            if (!(ok = wait(&sh.o_full[x], ns - 1))) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              uint32_t a[16];
              tmem_ld_32x32b_x16(t_o + c * 16, a);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 16; ++e) a[e] = __float_as_uint(__uint_as_float(a[e]) * f);
              tmem_st_32x32b_x16(t_o + c * 16, a);
            }
            tmem_st_wait();
          }
        }
        // ---- the weights
        const float shift = m == -INFINITY ? 0.0f : kTilesShift - m;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t a[32], w[16];
          tmem_ld_32x32b_x32(t_s + c * 32, a);
          tmem_ld_wait();
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const float4 sc = scales[c * 2 + g];
            const float by = factor(sc.x, qs), add = sc.y + shift;
            float part = 0.0f;
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              float z[2];
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                float acc = __uint_as_float(a[g * 16 + e + y]);
                if (!whole) {
                  const int32_t tok = c * 32 + g * 16 + e + y;
                  if (tok > last || tok < first) acc = -INFINITY;
                }
                z[y] = fast_exp2(fmaf(acc, by, add));
                part += z[y];
              }
              w[(g * 16 + e) / 2] = half2_of(z[0], z[1]);
            }
            sum = fmaf(part, sc.z, sum);
          }
          tmem_st_32x32b_x16(t_s + c * 16, w);
        }
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&sh.p_full[x]);
      }
      if (!ok) break;

      // ---- the output
      const bool mine = rows0 + row < it.rows;
      const int64_t out_row = (int64_t)(it.q0 + i) * (p.H * p.G) + it.h * p.G + j;
      const float inv = sum > 0.0f ? __fdividef(1.0f, sum) : (sum == 0.0f ? 0.0f : sum);
      if (it.tiles > 0) {
        if (!(ok = wait(&sh.o_full[x], ns - 1))) break;
        tc_fence_after();
      }
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t a[32];
        if (it.tiles > 0) {
          tmem_ld_32x32b_x32(t_o + c * 32, a);
          tmem_ld_wait();
        }
        if (mine) {
          uint4* dst = reinterpret_cast<uint4*>(p.out + out_row * D + c * 32);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float lo = it.tiles > 0 ? __uint_as_float(a[v * 8 + 2 * e]) * inv : 0.0f;
              const float hi = it.tiles > 0 ? __uint_as_float(a[v * 8 + 2 * e + 1]) * inv : 0.0f;
              w[e] = attend_pack2(p.fp16, lo, hi);
            }
            dst[v] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
      if (mine && p.lse)
        p.lse[out_row] = sum == 0.0f ? -INFINITY
                                     : (m - kTilesShift + log2f(sum)) * 0.69314718055994531f;
      tc_fence_before();
    }
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
  // At most an item for every pair of tiles that the batch's rows could fill.
  const int64_t rows = (int64_t)p.n_tokens * p.G;
  int64_t items = (rows / kPairRows + p.n_req) * p.H;
  if (items > num_sms()) items = num_sms();
  launch_pdl(kv_attend_tiles_kernel<D, FMT>, dim3((unsigned)items), dim3(kTilesThreads), smem,
             stream, p);
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "kv_attend_tiles launch");
}

}  // namespace

hs_status launch_kv_attend_tiles(const AttendParams& p, int32_t dim, int32_t format,
                                 cudaStream_t stream) {
  if (dim == 64)
    return format == HS_KV_E4M3 ? launch<64, HS_KV_E4M3>(p, stream)
                                : launch<64, HS_KV_INT8>(p, stream);
  return format == HS_KV_E4M3 ? launch<128, HS_KV_E4M3>(p, stream)
                              : launch<128, HS_KV_INT8>(p, stream);
}

}  // namespace hs
