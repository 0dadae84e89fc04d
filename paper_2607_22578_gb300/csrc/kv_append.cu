// New keys and values into the paged 8-bit cache (hs_kv_append).
//
// The batch's tokens of one block stand next to each other: a run.  For a run of c tokens that
// begins at offset o of block b, and each head,
//   m = the largest finite |x| of the run's c * dim values,
//   s = the least power of two >= 2^-126 with m <= C * s (C = 448 in e4m3, 127 in int8),
//   and where o > 0: s = max(s, the block's scale); if that grows, the o tokens' codes that are
//   there become round(code * old / s),
//   new codes = round(x / s), to nearest even, saturating.
// With scales that are powers of two, x / s is exact, so each value is rounded once (and an older
// code once more where its block's scale grows; in e4m3 that is exact but for subnormals).
//
// Every value is read once, every code written once: memory bounds it, and beside it the work on
// each value (65,536 x 8 x 128 keys and values 76 us, 5.2 TB/s, ALU pipe 71 %).  A CTA takes
// the runs that begin in its tile of tokens, for one head of K or V.  A run of few values (a
// decoding step's single tokens) is one warp's work, runs side by side; a longer one is the whole
// CTA's.  Either way its values stay in registers, 8 of a 16-byte load, between the maximum and
// the rounding.  128 threads a run of 8192 values: what is done once a warp weighs less than with
// 256 (147,000 tokens of 8 x 128, 212 -> 170 us), and with 64 too few loads are in flight (186);
// runs of 4096 values and fewer are shorter with 64 (6200 tokens of 5 x 64, 10.5 -> 8.0).
#include "kv_cache.cuh"

namespace hs {
namespace {

constexpr int kAppTile = 64;                  // tokens of a CTA, at most
constexpr int kAppFewTile = 4;                // ... in small batches
constexpr int kAppWindow = kAppTile + 128;    // with those that a run may reach past them
constexpr int kAppWarpVecs = 4;               // 16-byte pieces a lane of a run that a warp takes

struct AppendParams {
  uint8_t* k_codes;
  uint8_t* v_codes;
  float* k_scale;
  float* v_scale;
  const uint16_t* k;
  const uint16_t* v;
  int64_t n_blocks;
  int32_t H;
  int32_t bt_log2;
  int32_t dim;
  int64_t n_tokens;
  int64_t token_stride;
  int64_t head_stride;
  const int32_t* slots;
  int32_t tile;
  unsigned* err;
};

// 8 values from 16-bit storage, as floats
template <bool FP16>
__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (FP16) {
      const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      f[2 * i] = t.x;
      f[2 * i + 1] = t.y;
    } else {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

template <bool VEC>
__device__ __forceinline__ uint4 load8(const uint16_t* p) {
  if constexpr (VEC) {
    return __ldg(reinterpret_cast<const uint4*>(p));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (uint32_t)__ldg(p + 2 * i) | ((uint32_t)__ldg(p + 2 * i + 1) << 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// The largest magnitude of 8 values, as bits: of 16-bit floats without their sign, larger bits are
// larger numbers, and infinities and NaN are above all finite ones.
__device__ __forceinline__ uint32_t max_bits8(const uint4& v, uint32_t m) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = w[i] & 0x7fff7fffu;
    asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(a));
  }
  return m;
}

// ... and of the finite ones among them
__device__ __forceinline__ uint32_t max_finite_bits8(const uint4& v, uint32_t inf, uint32_t m) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
    m = max(m, max(lo < inf ? lo : 0u, hi < inf ? hi : 0u));
  }
  return m;
}

template <bool FP16>
__device__ __forceinline__ float magnitude(uint32_t bits) {
  return FP16 ? __half2float(__ushort_as_half((unsigned short)bits))
              : __uint_as_float(bits << 16);
}

// x / s.  A power of two is divided by exactly as a multiplication by its inverse.
struct Divisor {
  float s, inv;
  bool pow2;
  __device__ __forceinline__ explicit Divisor(float scale) : s(scale) {
    const uint32_t b = __float_as_uint(scale);
    pow2 = (b & 0x807fffffu) == 0 && b >= (1u << 23) && b <= (253u << 23);
    inv = pow2 ? __uint_as_float((254u << 23) - b) : 0.0f;
  }
  __device__ __forceinline__ float operator()(float x) const {
    return pow2 ? x * inv : __fdiv_rn(x, s);
  }
};

// PLAIN: the scale is a power of two and the values are finite, as they all but always are.
template <int FMT, bool FP16, bool PLAIN>
__device__ __forceinline__ uint2 encode8(const uint4& v, const Divisor& by) {
  float f[8];
  unpack8<FP16>(v, f);
  uint32_t h[4];
  if constexpr (PLAIN && FMT == HS_KV_INT8) {
    // |x / s| <= 127, so 1.5 * 2^23 + x / s has it, rounded to nearest even, in its low byte
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(fmaf(f[i], by.inv, 12582912.0f));
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __byte_perm(b[2 * i], b[2 * i + 1], 0x0040);
    return make_uint2(__byte_perm(h[0], h[1], 0x5410), __byte_perm(h[2], h[3], 0x5410));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      h[i] = PLAIN ? KvFormat<FMT>::encode2(f[2 * i] * by.inv, f[2 * i + 1] * by.inv)
                   : KvFormat<FMT>::encode2(by(f[2 * i]), by(f[2 * i + 1]));
    return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
  }
}

// n codes of a block (n a multiple of 16), times `ratio`, by `threads` threads of which this is
// number `me`.
template <int FMT>
__device__ __forceinline__ void rescale(uint8_t* codes, int n, float ratio, int me, int threads) {
  for (int i = me * 16; i < n; i += threads * 16) {
    uint4 v = *reinterpret_cast<const uint4*>(codes + i);
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t lo = KvFormat<FMT>::template decode2<0>(w[j]);
      const uint32_t hi = KvFormat<FMT>::template decode2<1>(w[j]);
      const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo));
      const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
      w[j] = KvFormat<FMT>::encode2(a.x * ratio, a.y * ratio) |
             (KvFormat<FMT>::encode2(b.x * ratio, b.y * ratio) << 16);
    }
    *reinterpret_cast<uint4*>(codes + i) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// NV: 16-byte pieces a thread holds of a run that the whole CTA takes, so that
// THREADS * NV * 8 values are a whole block.
template <int FMT, bool FP16, int THREADS, int NV, bool VEC>
__global__ void __launch_bounds__(THREADS, VEC ? (NV == 4 ? 10 : NV == 8 ? 8 : 512 / THREADS) : 1)
    kv_append_kernel(const AppendParams p) {
  constexpr int WARPS = THREADS / 32;
  __shared__ uint32_t begins[kAppWindow / 32];  // a bit for each token that ends the run before it
  __shared__ int32_t slot_s[kAppWindow];
  __shared__ uint32_t part[WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // The heads of a tile's tokens, keys and values, by CTAs that run together: a token's values are
  // read from one place of memory.
  const uint32_t heads = 2u * p.H, tile = blockIdx.x / heads, which = blockIdx.x - tile * heads;
  const bool keys = which < (uint32_t)p.H;
  const int h = keys ? which : which - p.H;
  const int64_t t0 = (int64_t)tile * p.tile;
  const uint16_t* x = (keys ? p.k : p.v) + h * p.head_stride;
  pdl_wait();
  pdl_trigger();
  for (int i = tid; i < kAppWindow; i += THREADS) {  // (whole warps)
    const int64_t t = t0 + i;
    const int32_t s = t < p.n_tokens ? __ldg(p.slots + t) : -1;
    const int32_t before = t > 0 && t <= p.n_tokens ? __ldg(p.slots + t - 1) : -1;
    // a run goes on within its block, one slot after the other
    const bool on = s >= 0 && before >= 0 && s == before + 1 &&
                    (s >> p.bt_log2) == (before >> p.bt_log2);
    const unsigned m = __ballot_sync(0xffffffffu, !on);
    slot_s[i] = s;
    if (lane == 0) begins[i >> 5] = m;
  }
  __syncthreads();

  // A run's 16-byte pieces, token by token: thread t's are THREADS apart, all of one column.
  const int row_log2 = 28 - __clz(p.dim);         // of the pieces of a token
  const int column = (tid & ((1 << row_log2) - 1)) * 8;
  const uint16_t* mine = x + (t0 + (tid >> row_log2)) * p.token_stride + column;
  const int64_t next_piece = (THREADS >> row_log2) * p.token_stride;
  constexpr uint32_t inf = FP16 ? 0x7c00u : 0x7f80u;
  int small = 0;
  for (int w = 0; w * 32 < p.tile; ++w) {
    for (uint32_t bits = begins[w]; bits; bits &= bits - 1) {
      const int i = w * 32 + __ffs(bits) - 1;
      if (i >= p.tile) break;
      const int32_t slot = slot_s[i];
      if (slot < 0) continue;
      const int64_t block = slot >> p.bt_log2;
      if (block >= p.n_blocks) {
        if (tid == 0) set_error(p.err, kErrInvalidArg);
        continue;
      }
      // where the next run begins, at most a block further on
      int next = i + 1;
      {
        int v = next >> 5;
        uint32_t rest = v < kAppWindow / 32 ? begins[v] & (0xffffffffu << (next & 31)) : 0u;
        while (rest == 0 && ++v < kAppWindow / 32) rest = begins[v];
        next = rest ? v * 32 + __ffs(rest) - 1 : kAppWindow;
      }
      const int off = slot & ((1 << p.bt_log2) - 1);
      const int pieces = (next - i) << row_log2;
      uint8_t* codes =
          (keys ? p.k_codes : p.v_codes) + ((block * p.H + h) << p.bt_log2) * p.dim;
      float* scale = (keys ? p.k_scale : p.v_scale) + block * p.H + h;
      if (pieces <= 32 * kAppWarpVecs) {
        if ((small++ & (WARPS - 1)) != warp) continue;
        const uint16_t* src = x + (t0 + i + (lane >> row_log2)) * p.token_stride +
                              (lane & ((1 << row_log2) - 1)) * 8;
        uint4 v[kAppWarpVecs];
        const float old = off > 0 ? *scale : 0.0f;
        uint32_t m = 0u;
#pragma unroll
        for (int k = 0; k < kAppWarpVecs; ++k) {
          v[k] = k * 32 + lane < pieces ? load8<VEC>(src + k * (32 >> row_log2) * p.token_stride)
                                        : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int k = 0; k < kAppWarpVecs; ++k) m = max_bits8(v[k], m);
        m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
        const bool finite = m < inf;
        if (!finite) {
          m = 0u;
#pragma unroll
          for (int k = 0; k < kAppWarpVecs; ++k) m = max_finite_bits8(v[k], inf, m);
          m = __reduce_max_sync(0xffffffffu, m);
        }
        const float s = fmaxf(kv_scale<FMT>(magnitude<FP16>(m)), old);
        if (off > 0 && s > old)
          rescale<FMT>(codes, off * p.dim, __fdiv_rn(old, s), lane, 32);
        const Divisor by(s);
        const bool plain = finite && by.pow2;
#pragma unroll
        for (int k = 0; k < kAppWarpVecs; ++k) {
          const int j = k * 32 + lane;
          if (j < pieces)
            *reinterpret_cast<uint2*>(codes + off * p.dim + j * 8) =
                plain ? encode8<FMT, FP16, true>(v[k], by) : encode8<FMT, FP16, false>(v[k], by);
        }
        if (lane == 0) *scale = s;
        continue;
      }
      uint4 v[NV];
      const float old = off > 0 ? *scale : 0.0f;
      uint32_t m = 0u;
      const uint16_t* src = mine + i * p.token_stride;
#pragma unroll
      for (int k = 0; k < NV; ++k)
        v[k] = k * THREADS + tid < pieces ? load8<VEC>(src + k * next_piece)
                                              : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int k = 0; k < NV; ++k) m = max_bits8(v[k], m);
      m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
      if (lane == 0) part[warp] = m;
      __syncthreads();                            // also: everyone has read the old scale
#pragma unroll
      for (int k = 0; k < WARPS; ++k) m = max(m, part[k]);
      const bool finite = m < inf;
      if (!finite) {
        __syncthreads();
        m = 0u;
#pragma unroll
        for (int k = 0; k < NV; ++k) m = max_finite_bits8(v[k], inf, m);
        m = __reduce_max_sync(0xffffffffu, m);
        if (lane == 0) part[warp] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < WARPS; ++k) m = max(m, part[k]);
      }
      const float s = fmaxf(kv_scale<FMT>(magnitude<FP16>(m)), old);
      if (off > 0 && s > old)
        rescale<FMT>(codes, off * p.dim, __fdiv_rn(old, s), tid, THREADS);
      const Divisor by(s);
      uint8_t* dst = codes + off * p.dim + tid * 8;
      if (finite && by.pow2) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (k * THREADS + tid < pieces)
            *reinterpret_cast<uint2*>(dst + k * THREADS * 8) =
                encode8<FMT, FP16, true>(v[k], by);
      } else {
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (k * THREADS + tid < pieces)
            *reinterpret_cast<uint2*>(dst + k * THREADS * 8) =
                encode8<FMT, FP16, false>(v[k], by);
      }
      if (tid == 0) *scale = s;
      __syncthreads();                            // `part` is free again
    }
  }
}

template <int FMT, bool FP16, int THREADS, int NV>
hs_status launch(const AppendParams& p, bool vec, dim3 grid, cudaStream_t stream) {
  launch_pdl(vec ? kv_append_kernel<FMT, FP16, THREADS, NV, true>
                 : kv_append_kernel<FMT, FP16, THREADS, NV, false>,
             grid, dim3(THREADS), 0, stream, p);
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "kv_append launch");
}

template <int FMT, bool FP16>
hs_status launch_pieces(const AppendParams& p, bool vec, dim3 grid, cudaStream_t stream) {
  const int pieces = (p.dim << p.bt_log2) / 8;  // of a block: 128 to 4096
  if (pieces <= 64 * 8) return launch<FMT, FP16, 64, 8>(p, vec, grid, stream);
  if (pieces <= 128 * 8) return launch<FMT, FP16, 128, 8>(p, vec, grid, stream);
  if (pieces <= 128 * 16) return launch<FMT, FP16, 128, 16>(p, vec, grid, stream);
  return launch<FMT, FP16, 256, 16>(p, vec, grid, stream);
}

template <int FMT>
hs_status launch_format(const AppendParams& p, int32_t dtype, bool vec, dim3 grid,
                        cudaStream_t stream) {
  return dtype == HS_KV_FP16 ? launch_pieces<FMT, true>(p, vec, grid, stream)
                             : launch_pieces<FMT, false>(p, vec, grid, stream);
}

}  // namespace

hs_status launch_kv_append(const hs_kv_cache& c, int32_t bt_log2, const uint16_t* k,
                           const uint16_t* v, int32_t dtype, int64_t n_tokens,
                           int64_t token_stride, int64_t head_stride, const int32_t* slots,
                           cudaStream_t stream) {
  unsigned* err = device_error_word();
  if (!err) return fail(HS_ERR_CUDA, "could not resolve the device error word");
  AppendParams p{};
  p.k_codes = static_cast<uint8_t*>(c.k);
  p.v_codes = static_cast<uint8_t*>(c.v);
  p.k_scale = c.k_scale;
  p.v_scale = c.v_scale;
  p.k = k;
  p.v = v;
  p.n_blocks = c.n_blocks;
  p.H = c.n_kv_heads;
  p.bt_log2 = bt_log2;
  p.dim = c.dim;
  p.n_tokens = n_tokens;
  p.token_stride = token_stride;
  p.head_stride = head_stride;
  p.slots = slots;
  p.err = err;
  // Some twelve CTAs an SM: larger tiles leave SMs without work, smaller ones mean more CTAs.  64
  // lone tokens of 8 heads: 4.0 us with tiles of 4, 38 with 64; 2000 in whole blocks: 12.7 and 8.6,
  // 6.6 with 32; 16,000: 91 and 36.
  const int64_t per_sm = (n_tokens * c.n_kv_heads * 2 + num_sms() - 1) / num_sms();
  p.tile = kAppFewTile;
  while (p.tile < kAppTile && per_sm > 12 * p.tile) p.tile *= 2;
  const int64_t tiles = (n_tokens + p.tile - 1) / p.tile;
  const bool vec = token_stride % 8 == 0 && head_stride % 8 == 0 &&
                   reinterpret_cast<uintptr_t>(k) % 16 == 0 &&
                   reinterpret_cast<uintptr_t>(v) % 16 == 0;
  const int64_t ctas = tiles * c.n_kv_heads * 2;
  if (ctas > 0x7fffffffLL) return fail(HS_ERR_UNSUPPORTED, "n_tokens * n_kv_heads too large");
  const dim3 grid((unsigned)ctas);
  return c.format == HS_KV_E4M3 ? launch_format<HS_KV_E4M3>(p, dtype, vec, grid, stream)
                                : launch_format<HS_KV_INT8>(p, dtype, vec, grid, stream);
}

}  // namespace hs
