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
// Every value is read once, every code written once: the kernel is bound by memory.  A CTA takes
// the runs that begin in its tile of tokens, for one head of K or V.  A run of few values (a
// decoding step's single tokens) is one warp's work, runs side by side; a longer one is the whole
// CTA's.  Either way its values stay in registers, 8 of a 16-byte load, between the maximum and
// the rounding.
#include "kv_cache.cuh"

namespace hs {
namespace {

constexpr int kAppThreads = 256;
constexpr int kAppWarps = kAppThreads / 32;
constexpr int kAppTile = 64;                  // tokens of a CTA, at most
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
  int32_t fp16;
  int64_t n_tokens;
  int64_t token_stride;
  int64_t head_stride;
  const int32_t* slots;
  int32_t tile;
  unsigned* err;
};

// 8 values from 16-bit storage, as floats
__device__ __forceinline__ void unpack8(const uint4& v, int fp16, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (fp16) {
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

__device__ __forceinline__ float finite_max8(const uint4& v, int fp16, float m) {
  float f[8];
  unpack8(v, fp16, f);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(f[i]);
    m = fmaxf(m, a <= 3.4028234663852886e38f ? a : 0.0f);  // not of NaN and infinities
  }
  return m;
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

template <int FMT>
__device__ __forceinline__ uint2 encode8(const uint4& v, int fp16, const Divisor& by) {
  float f[8];
  unpack8(v, fp16, f);
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = KvFormat<FMT>::encode2(by(f[2 * i]), by(f[2 * i + 1]));
  return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
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
// kAppThreads * NV * 8 values are a whole block.
template <int FMT, int NV, bool VEC>
__global__ void __launch_bounds__(kAppThreads) kv_append_kernel(const AppendParams p) {
  __shared__ uint32_t begins[kAppWindow / 32];  // a bit for each token that ends the run before it
  __shared__ int32_t slot_s[kAppWindow];
  __shared__ float part[kAppWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = blockIdx.y;
  const bool keys = blockIdx.z == 0;
  const int64_t t0 = (int64_t)blockIdx.x * p.tile;
  pdl_wait();
  pdl_trigger();
  if (tid < kAppWindow) {
    const int64_t t = t0 + tid;
    const int32_t s = t < p.n_tokens ? __ldg(p.slots + t) : -1;
    const int32_t before = t > 0 && t <= p.n_tokens ? __ldg(p.slots + t - 1) : -1;
    // a run goes on within its block, one slot after the other
    const bool on = s >= 0 && before >= 0 && s == before + 1 &&
                    (s >> p.bt_log2) == (before >> p.bt_log2);
    const unsigned m = __ballot_sync(0xffffffffu, !on);
    slot_s[tid] = s;
    if (lane == 0) begins[tid >> 5] = m;
  }
  __syncthreads();

  const uint16_t* x = (keys ? p.k : p.v) + h * p.head_stride;
  const int per_row = p.dim >> 3;                 // pieces of a token
  const int row_log2 = 31 - __clz(per_row);
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
      const uint16_t* xr = x + (t0 + i) * p.token_stride;
      const auto piece = [&](int j) {
        return load8<VEC>(xr + (j >> row_log2) * p.token_stride + (j & (per_row - 1)) * 8);
      };
      if (pieces <= 32 * kAppWarpVecs) {
        if ((small++ & (kAppWarps - 1)) != warp) continue;
        uint4 v[kAppWarpVecs];
        const float old = off > 0 ? *scale : 0.0f;
        float m = 0.0f;
#pragma unroll
        for (int k = 0; k < kAppWarpVecs; ++k) {
          const int j = k * 32 + lane;
          v[k] = j < pieces ? piece(j) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int k = 0; k < kAppWarpVecs; ++k) m = finite_max8(v[k], p.fp16, m);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float s = fmaxf(kv_scale<FMT>(m), old);
        if (off > 0 && s > old)
          rescale<FMT>(codes, off * p.dim, __fdiv_rn(old, s), lane, 32);
        const Divisor by(s);
#pragma unroll
        for (int k = 0; k < kAppWarpVecs; ++k) {
          const int j = k * 32 + lane;
          if (j < pieces)
            *reinterpret_cast<uint2*>(codes + off * p.dim + j * 8) =
                encode8<FMT>(v[k], p.fp16, by);
        }
        if (lane == 0) *scale = s;
        continue;
      }
      uint4 v[NV];
      const float old = off > 0 ? *scale : 0.0f;
      float m = 0.0f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int j = k * kAppThreads + tid;
        v[k] = j < pieces ? piece(j) : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) m = finite_max8(v[k], p.fp16, m);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      if (lane == 0) part[warp] = m;
      __syncthreads();                            // also: everyone has read the old scale
#pragma unroll
      for (int k = 0; k < kAppWarps; ++k) m = fmaxf(m, part[k]);
      const float s = fmaxf(kv_scale<FMT>(m), old);
      if (off > 0 && s > old)
        rescale<FMT>(codes, off * p.dim, __fdiv_rn(old, s), tid, kAppThreads);
      const Divisor by(s);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int j = k * kAppThreads + tid;
        if (j < pieces)
          *reinterpret_cast<uint2*>(codes + off * p.dim + j * 8) = encode8<FMT>(v[k], p.fp16, by);
      }
      if (tid == 0) *scale = s;
      __syncthreads();                            // `part` is free again
    }
  }
}

template <int FMT, int NV>
hs_status launch(const AppendParams& p, bool vec, dim3 grid, cudaStream_t stream) {
  launch_pdl(vec ? kv_append_kernel<FMT, NV, true> : kv_append_kernel<FMT, NV, false>, grid,
             dim3(kAppThreads), 0, stream, p);
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "kv_append launch");
}

template <int FMT>
hs_status launch_format(const AppendParams& p, bool vec, dim3 grid, cudaStream_t stream) {
  const int pieces = (p.dim << p.bt_log2) / 8;  // of a block: 128 to 4096
  if (pieces <= kAppThreads * 4) return launch<FMT, 4>(p, vec, grid, stream);
  if (pieces <= kAppThreads * 8) return launch<FMT, 8>(p, vec, grid, stream);
  return launch<FMT, 16>(p, vec, grid, stream);
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
  p.fp16 = dtype == HS_KV_FP16;
  p.n_tokens = n_tokens;
  p.token_stride = token_stride;
  p.head_stride = head_stride;
  p.slots = slots;
  p.err = err;
  // Small batches: few tokens a CTA, so that every SM has some.
  const int64_t per_sm = (n_tokens * c.n_kv_heads * 2 + num_sms() - 1) / num_sms();
  p.tile = per_sm >= 4 * kAppTile ? kAppTile : kAppWarps;
  const int64_t tiles = (n_tokens + p.tile - 1) / p.tile;
  const bool vec = token_stride % 8 == 0 && head_stride % 8 == 0 &&
                   reinterpret_cast<uintptr_t>(k) % 16 == 0 &&
                   reinterpret_cast<uintptr_t>(v) % 16 == 0;
  const dim3 grid((unsigned)tiles, (unsigned)c.n_kv_heads, 2);
  return c.format == HS_KV_E4M3 ? launch_format<HS_KV_E4M3>(p, vec, grid, stream)
                                : launch_format<HS_KV_INT8>(p, vec, grid, stream);
}

}  // namespace hs
