// What the kernels of hs_kv_attend share: their arguments, a request's place, 16-bit values.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hs_internal.cuh"

namespace hs {

struct AttendParams {
  const uint8_t* k;
  const uint8_t* v;
  const float* ks;
  const float* vs;
  int32_t n_blocks;
  int32_t H;                 // kv heads
  int32_t G;                 // query heads of each
  uint32_t G_inv;            // ceil(2^32 / G), or 0: see attend_query
  int32_t bt_log2;
  const uint16_t* q;
  int64_t q_token, q_head;   // strides, in elements
  int32_t q_vec;             // rows of q are 16-byte aligned
  int32_t fp16;
  int32_t n_tokens;
  int32_t max_q;
  const int32_t* lens;
  const int32_t* starts;     // or NULL: max_q queries each
  int32_t n_req;
  const int32_t* n_req_dev;
  const int32_t* table;
  int32_t width;
  int32_t causal;
  int32_t window;
  int32_t rows_most;         // requests with more rows (queries times G) are another kernel's
  int32_t apart;             // the other kernel runs before this one on the stream
  float scale_log2;          // scale * log2(e)
  uint16_t* out;
  float* lse;
  unsigned* counters;
  unsigned* queue;           // of the kernel of many rows: items drawn, CTAs that are done
  float* partial;
  unsigned* tile_counters;   // of the kernel of many rows: parts done of each warp's rows of an item
  float* tile_partial;
  unsigned* err;
};

constexpr int kAttendMaxPerSm = 4;  // CTAs of a launch that one SM holds, at most

// A counter for each CTA of a launch, the queue's two, and eight for each SM's item.
inline int64_t attend_counters() { return (int64_t)num_sms() * kAttendMaxPerSm; }
inline int64_t attend_counter_bytes() {
  return ((attend_counters() + 2 + num_sms() * 8) * 4 + 255) / 256 * 256;
}

// Request r's queries (n of them, from token q0 of the batch) and tokens in the cache; false if
// it has none, or its numbers cannot be (*bad).
__device__ __forceinline__ bool attend_request(const AttendParams& p, int32_t r, int32_t& n,
                                               int32_t& q0, int32_t& len, unsigned* bad) {
  if (p.starts) {
    q0 = __ldg(p.starts + r);
    const int64_t m = (int64_t)__ldg(p.starts + r + 1) - q0;
    n = (int32_t)(m < -1 ? -1 : (m > 0x7fffffffLL ? 0x7fffffffLL : m));
  } else {
    n = p.max_q;
    q0 = r * p.max_q;
  }
  len = __ldg(p.lens + r);
  if (n == 0) return false;
  if (n < 0 || n > p.max_q || q0 < 0 || q0 > p.n_tokens - n || len < 0 ||
      len > ((int64_t)p.width << p.bt_log2)) {
    *bad = kErrInvalidArg;
    return false;
  }
  return true;
}

// A request's window: one longer than what it has hides nothing, and so 31 bits hold a position less
// it, also of queries (2^30 at most) that stand before the first token.
__device__ __forceinline__ int32_t attend_window(const AttendParams& p, int32_t len) {
  return min(p.window, len);
}

// The first token that a query of a request sees.  What is before it is loaded as zeros: a weight of 0
// would not keep a NaN among its values from the outputs.
__device__ __forceinline__ int32_t attend_first(const AttendParams& p, int32_t n, int32_t len) {
  return p.window > 0 ? max(len - n - attend_window(p, len) + 1, 0) : 0;
}

static __device__ __noinline__ int32_t attend_divide(int32_t row, int32_t G) { return row / G; }

// The query that a request's row belongs to: row / G.  With m = ceil(2^32 / G), m * G is less than
// G over 2^32, so row * m / 2^32 is exact while row * G < 2^32; the host gives m where every row is
// and G > 1.  The division itself stands out of line.
__device__ __forceinline__ int32_t attend_query(const AttendParams& p, int32_t row) {
  if (p.G_inv) return (int32_t)__umulhi((uint32_t)row, p.G_inv);
  return p.G == 1 ? row : attend_divide(row, p.G);
}

// 8 values of 16 bits that are only 2-byte aligned
static __device__ __noinline__ uint4 attend_raw8(const uint16_t* src) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = (uint32_t)__ldg(src + 2 * i) | ((uint32_t)__ldg(src + 2 * i + 1) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float2 attend_unpack2(uint32_t w, int fp16) {
  if (fp16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

__device__ __forceinline__ void attend_unpack8(const uint4& v, int fp16, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 t = attend_unpack2(w[i], fp16);
    f[2 * i] = t.x;
    f[2 * i + 1] = t.y;
  }
}

// cp.async of 16 bytes, or of as many zeros
__device__ __forceinline__ void cp_async16_zfill(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
               "r"(in ? 16 : 0)
               : "memory");
}

// 2^x to 2 units in the last place; below the normal range 0
__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two neighbouring outputs, rounded to nearest even
__device__ __forceinline__ uint32_t attend_pack2(int fp16, float x0, float x1) {
  if (fp16) {
    const __half2 h = __floats2half2_rn(x0, x1);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(x0, x1);
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace hs
