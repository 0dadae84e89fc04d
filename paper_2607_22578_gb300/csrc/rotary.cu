// Rotary positions (hs_rotary): pair i of every head of a token at position p becomes
//   (m (a cos t - b sin t), m (b cos t + a sin t)),  t = 2 pi * (p * turns[i] / 2^64),
// with -t for the way back (the transpose, so the gradient).  turns[i] is a fraction of a turn in
// 64 bits, so p * turns[i] mod 2^64 is the angle without its whole turns, exactly, however far p
// is: what an angle in 32-bit floats loses at position 100,000 (2^-7 of a radian) never arises.
// Its eighths of a turn choose the octant, the rest (at most pi / 4) goes through Taylor's series.
//
// Memory bounds it: each value is read and written once.  A thread keeps the sines and cosines of
// some pairs of one token in registers and goes over heads with them.  18,400 tokens of 40 heads of
// 128 (94 M values, 56 us at the copy rate): 63 us interleaved, 66 in halves of whole pieces, 75 in
// halves of 45; a pair a thread, as where heads are no whole pieces of 16 bytes, takes 130, and 203 in
// place: its loads and stores are 2 bytes a lane, and heads with gaps leave sectors written in part.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "rotary.cuh"

namespace hs {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotPairs = 8;  // pairs of a thread: two 16-byte pieces

// The request of token t, by a whole warp: the last r < R with starts[r] <= t, or -1.
__device__ __forceinline__ int32_t find_request(const int32_t* starts, int32_t R, int32_t t) {
  const int lane = threadIdx.x & 31;
  int32_t lo = 0, n = R;
  while (n > 0) {
    const int32_t step = (n + 31) / 32;
    const int32_t at = lane * step;
    const bool le = at < n && __ldg(starts + lo + at) <= t;
    const int c = __popc(__ballot_sync(0xffffffffu, le));
    if (c == 0) return -1;  // (only in the first round)
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
    if (step == 1) break;
  }
  return n > 0 ? lo : -1;
}

// cos and sin of 2 pi * phase / 2^64, times m.
__device__ __forceinline__ void turn(uint64_t phase, float m, float& c, float& s) {
  const uint32_t u = (uint32_t)((phase + 0x80000000ull) >> 32);
  const uint32_t q = (u + 0x20000000u) >> 30;  // the nearest quarter turn
  const float x = (float)(int32_t)(u - (q << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float y = x * x;
  // to x^9 / 9! and x^10 / 10! : the next terms are below 2^-29 and 2^-33 at pi / 4
  float a = fmaf(y, 2.7557319224e-6f, -1.9841269841e-4f);
  a = fmaf(y, a, 8.3333333333e-3f);
  a = fmaf(y, a, -1.6666666667e-1f);
  a = fmaf(x * y, a, x);
  float b = fmaf(y, -2.7557319224e-7f, 2.4801587302e-5f);
  b = fmaf(y, b, -1.3888888889e-3f);
  b = fmaf(y, b, 4.1666666667e-2f);
  b = fmaf(y, b, -0.5f);
  b = fmaf(y, b, 1.0f);
  const float cc = (q & 1) ? a : b, ss = (q & 1) ? b : a;
  c = ((q + 1) & 2) ? -m * cc : m * cc;
  s = (q & 2) ? -m * ss : m * ss;
}

template <bool FP16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (FP16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

template <bool FP16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  if constexpr (FP16) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}

template <bool FP16>
__device__ __forceinline__ float unpack1(uint16_t w) {
  if constexpr (FP16) return __half2float(__ushort_as_half(w));
  return __uint_as_float((uint32_t)w << 16);
}

template <bool FP16>
__device__ __forceinline__ uint16_t pack1(float x) {
  if constexpr (FP16) return __half_as_ushort(__float2half_rn(x));
  return __bfloat16_as_ushort(__float2bfloat16_rn(x));
}

// Positions of the CTA's tokens into shared memory; ok says which have one.
__device__ __forceinline__ void positions(const RotaryParams& p, int32_t t0, int32_t n,
                                          int32_t* pos, uint8_t* ok) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t R = p.n_req;
  if (p.n_req_dev) {
    const int32_t c = __ldg(p.n_req_dev);
    R = c < 0 ? 0 : c < R ? c : R;
  }
  if (p.positions) {
    for (int32_t i = threadIdx.x; i < n; i += kRotThreads) {
      pos[i] = __ldg(p.positions + t0 + i);
      ok[i] = 1;
    }
  } else {
    for (int32_t i = warp; i < n; i += kRotThreads / 32) {
      const int32_t t = t0 + i, r = find_request(p.starts, R, t);
      if (lane == 0) {
        bool good = false;
        if (r >= 0) {
          const int32_t a = __ldg(p.starts + r), b = __ldg(p.starts + r + 1);
          const int32_t len = __ldg(p.lens + r);
          if (a < 0 || b < a || b > p.n_tokens || len < b - a) {
            set_error(p.err, kErrInvalidArg);
          } else if (t < b) {  // (else it is behind the last request's)
            good = true;
            pos[i] = len - b + t;
          }
        }
        ok[i] = good;
      }
    }
  }
  __syncthreads();
}

// 16 values of a head: 8 pairs, or 16 values that are not turned.  Halves of whole pieces, or
// interleaved in heads of more than 256.
template <bool FP16, bool HALF>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const RotaryParams p) {
  __shared__ int32_t pos[kRotThreads];
  __shared__ uint8_t ok[kRotThreads];
  pdl_wait();
  pdl_trigger();
  const int32_t units = p.dim / 16, turned = p.rot / 16;
  const int32_t per = max(1, kRotThreads / units);  // tokens of the CTA
  const int32_t t0 = blockIdx.x * per, n = min(per, p.n_tokens - t0);
  positions(p, t0, n, pos, ok);
  const int32_t h0 = blockIdx.y * p.heads_per, h1 = min(h0 + p.heads_per, p.H);
  for (int32_t at = threadIdx.x; at < n * units; at += kRotThreads) {
    const int32_t i = at / units, u = at - i * units;
    if (!ok[i]) continue;
    const bool turns = u < turned;
    if (!turns && p.in_place) continue;
    float c[kRotPairs], s[kRotPairs];
    if (turns) {
      const int64_t ps = p.inverse ? -(int64_t)pos[i] : (int64_t)pos[i];
#pragma unroll
      for (int j = 0; j < kRotPairs; ++j)
        turn((uint64_t)ps * __ldg(p.turns + u * kRotPairs + j), p.magnitude, c[j], s[j]);
    }
    const int32_t e0 = HALF && turns ? u * 8 : u * 16;
    const int32_t e1 = HALF && turns ? p.rot / 2 + u * 8 : u * 16 + 8;
    const uint16_t* x = p.x + (int64_t)(t0 + i) * p.x_token + h0 * p.x_head;
    uint16_t* y = p.out + (int64_t)(t0 + i) * p.out_token + h0 * p.out_head;
    // Two heads' loads on the way together (out may be x, so that a store holds up later loads).
    for (int32_t h = h0; h < h1; h += 2, x += 2 * p.x_head, y += 2 * p.out_head) {
      uint4 v[2][2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (h + q >= h1) break;
        v[q][0] = *reinterpret_cast<const uint4*>(x + q * p.x_head + e0);
        v[q][1] = *reinterpret_cast<const uint4*>(x + q * p.x_head + e1);
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (h + q >= h1) break;
        if (turns) {
          uint32_t w[8] = {v[q][0].x, v[q][0].y, v[q][0].z, v[q][0].w,
                           v[q][1].x, v[q][1].y, v[q][1].z, v[q][1].w};
          if constexpr (HALF) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 a = unpack2<FP16>(w[j]), b = unpack2<FP16>(w[j + 4]);
              w[j] = pack2<FP16>(fmaf(a.x, c[2 * j], -(b.x * s[2 * j])),
                                 fmaf(a.y, c[2 * j + 1], -(b.y * s[2 * j + 1])));
              w[j + 4] = pack2<FP16>(fmaf(b.x, c[2 * j], a.x * s[2 * j]),
                                     fmaf(b.y, c[2 * j + 1], a.y * s[2 * j + 1]));
            }
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float2 a = unpack2<FP16>(w[j]);
              w[j] = pack2<FP16>(fmaf(a.x, c[j], -(a.y * s[j])), fmaf(a.y, c[j], a.x * s[j]));
            }
          }
          v[q][0] = make_uint4(w[0], w[1], w[2], w[3]);
          v[q][1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
        *reinterpret_cast<uint4*>(y + q * p.out_head + e0) = v[q][0];
        *reinterpret_cast<uint4*>(y + q * p.out_head + e1) = v[q][1];
      }
    }
  }
}

// Any rot, for heads of whole 16-byte pieces (32 at most): a lane a piece, a warp one or more
// tokens, one head of each at a time.  The other value of a pair lies anywhere in the same head,
// which the warp holds in shared memory while it turns it (so out may be x here too).
template <bool FP16, bool HALF>
__global__ void __launch_bounds__(kRotThreads) rotary_rows_kernel(const RotaryParams p) {
  __shared__ int32_t pos[kRotThreads];
  __shared__ uint8_t ok[kRotThreads];
  __shared__ uint4 held[kRotThreads / 32][2][32];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t units = p.dim / 8, rows = 32 / units;
  const int32_t per = kRotThreads / 32 * rows;  // tokens of the CTA
  const int32_t t0 = blockIdx.x * per, n = min(per, p.n_tokens - t0);
  positions(p, t0, n, pos, ok);
  const int32_t row = lane / units, u = lane - row * units, i = warp * rows + row;
  const bool on = row < rows && i < n && ok[i];
  const int32_t half = p.rot / 2, e = u * 8;
  const bool moves = on && (e < p.rot || !p.in_place);
  float c[8], s[8];
  int32_t other[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    c[j] = s[j] = 0.0f;
    other[j] = lane * 8 + j;
    if (!on || e + j >= p.rot || (!HALF && (j & 1))) continue;
    const bool second = HALF && e + j >= half;
    const int32_t pair = HALF ? e + j - (second ? half : 0) : (e + j) / 2;
    const int64_t ps = p.inverse ? -(int64_t)pos[i] : (int64_t)pos[i];
    turn((uint64_t)ps * __ldg(p.turns + pair), p.magnitude, c[j], s[j]);
    if (HALF) {
      other[j] += second ? -half : half;
      if (!second) s[j] = -s[j];
    }
  }
  const int32_t h0 = blockIdx.y * p.heads_per, h1 = min(h0 + p.heads_per, p.H);
  const uint16_t* x = p.x + (int64_t)(t0 + i) * p.x_token + h0 * p.x_head + e;
  uint16_t* y = p.out + (int64_t)(t0 + i) * p.out_token + h0 * p.out_head + e;
  for (int32_t h = h0; h < h1; h += 2, x += 2 * p.x_head, y += 2 * p.out_head) {
    uint4 v[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      v[q] = make_uint4(0, 0, 0, 0);
      if (on && h + q < h1) v[q] = *reinterpret_cast<const uint4*>(x + q * p.x_head);
      if (HALF) held[warp][q][lane] = v[q];
    }
    if (HALF) __syncwarp();
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      uint32_t w[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
      const uint16_t* head = reinterpret_cast<const uint16_t*>(held[warp][q]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 a = unpack2<FP16>(w[j]);
        uint32_t turned;
        if constexpr (HALF)
          turned = pack2<FP16>(fmaf(a.x, c[2 * j], unpack1<FP16>(head[other[2 * j]]) * s[2 * j]),
                               fmaf(a.y, c[2 * j + 1],
                                    unpack1<FP16>(head[other[2 * j + 1]]) * s[2 * j + 1]));
        else
          turned = pack2<FP16>(fmaf(a.x, c[2 * j], -(a.y * s[2 * j])),
                               fmaf(a.y, c[2 * j], a.x * s[2 * j]));
        // (rot is even: both of a word are turned, or neither)
        if (e + 2 * j < p.rot) w[j] = turned;
      }
      if (moves && h + q < h1)
        *reinterpret_cast<uint4*>(y + q * p.out_head) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (HALF) __syncwarp();  // (the next heads go where these are still read)
  }
}

// Any dim, rot and strides: a pair, or a value that is not turned, at a time.
template <bool FP16>
__global__ void __launch_bounds__(kRotThreads) rotary_any_kernel(const RotaryParams p) {
  __shared__ int32_t pos[kRotThreads];
  __shared__ uint8_t ok[kRotThreads];
  pdl_wait();
  pdl_trigger();
  const int32_t half = p.rot / 2, units = p.in_place ? half : half + p.dim - p.rot;
  const int32_t per = max(1, kRotThreads / units);
  const int32_t t0 = blockIdx.x * per, n = min(per, p.n_tokens - t0);
  positions(p, t0, n, pos, ok);
  const int32_t h0 = blockIdx.y * p.heads_per, h1 = min(h0 + p.heads_per, p.H);
  for (int32_t at = threadIdx.x; at < n * units; at += kRotThreads) {
    const int32_t i = at / units, u = at - i * units;
    if (!ok[i]) continue;
    const uint16_t* x = p.x + (int64_t)(t0 + i) * p.x_token + h0 * p.x_head;
    uint16_t* y = p.out + (int64_t)(t0 + i) * p.out_token + h0 * p.out_head;
    if (u >= half) {
      const int32_t e = p.rot + u - half;
      for (int32_t h = h0; h < h1; ++h, x += p.x_head, y += p.out_head) y[e] = x[e];
      continue;
    }
    const int64_t ps = p.inverse ? -(int64_t)pos[i] : (int64_t)pos[i];
    float c, s;
    turn((uint64_t)ps * __ldg(p.turns + u), p.magnitude, c, s);
    const int32_t e0 = p.half ? u : 2 * u, e1 = p.half ? u + half : 2 * u + 1;
    for (int32_t h = h0; h < h1; ++h, x += p.x_head, y += p.out_head) {
      const float a = unpack1<FP16>(x[e0]), b = unpack1<FP16>(x[e1]);
      y[e0] = pack1<FP16>(fmaf(a, c, -(b * s)));
      y[e1] = pack1<FP16>(fmaf(b, c, a * s));
    }
  }
}

}  // namespace

hs_status launch_rotary(RotaryParams p, bool pieces, bool fp16, cudaStream_t stream) {
  p.err = device_error_word();
  if (!p.err) return fail(HS_ERR_CUDA, "could not resolve the device error word");
  // By lanes of a piece each, or where both halves are whole pieces by threads that hold both (66 us
  // and not 75 for the size above), or a pair at a time.
  const bool whole = p.dim % 16 == 0 && p.rot % 16 == 0;
  const bool rows = pieces && p.dim % 8 == 0 && p.dim <= 256 && !(whole && p.half);
  const bool vec = pieces && whole && !rows;
  int32_t per;  // tokens of a CTA
  if (rows) {
    per = kRotThreads / 32 * (32 / (p.dim / 8));
  } else {
    const int32_t units = vec ? p.dim / 16 : p.in_place ? p.rot / 2 : p.rot / 2 + p.dim - p.rot;
    per = units < kRotThreads ? kRotThreads / units : 1;
  }
  const int64_t grid = ((int64_t)p.n_tokens + per - 1) / per;
  // Heads of a thread: as many as leave every SM a few CTAs, so that sines are taken seldom.
  int32_t heads = rows ? 16 : 8;
  while (heads > 1 && grid * ((p.H + heads - 1) / heads) < 4 * num_sms()) heads /= 2;
  while ((p.H + heads - 1) / heads > 65535) heads *= 2;
  const int32_t shares = (p.H + heads - 1) / heads;
  heads = (p.H + shares - 1) / shares;
  p.heads_per = heads;
  const dim3 blocks((unsigned)grid, (unsigned)((p.H + heads - 1) / heads));
  const dim3 threads(kRotThreads);
  if (rows && p.half) {
    launch_pdl(fp16 ? rotary_rows_kernel<true, true> : rotary_rows_kernel<false, true>, blocks,
               threads, 0, stream, p);
  } else if (rows) {
    launch_pdl(fp16 ? rotary_rows_kernel<true, false> : rotary_rows_kernel<false, false>, blocks,
               threads, 0, stream, p);
  } else if (!vec) {
    launch_pdl(fp16 ? rotary_any_kernel<true> : rotary_any_kernel<false>, blocks, threads, 0,
               stream, p);
  } else if (p.half) {
    launch_pdl(fp16 ? rotary_kernel<true, true> : rotary_kernel<false, true>, blocks, threads, 0,
               stream, p);
  } else {
    launch_pdl(fp16 ? rotary_kernel<true, false> : rotary_kernel<false, false>, blocks, threads, 0,
               stream, p);
  }
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "rotary launch");
}

}  // namespace hs
