// Draws of tokens (hs_sample): temperature, top-k, top-p, min-p and one given uniform number.
//
// With a row's logits in order (the largest first, equal ones by index) and weights
// w = exp((l - l_max) / T), each filter keeps a prefix of that order, and the token is the first
// whose sum of weights C_m exceeds u * W, W the weights' sum of what is kept.  Sums are whole
// numbers of 2^-43 of the largest weight, of weights from an exponential in pairs of floats that is
// right to 2^-42, so they do not depend on the order of anything, and a draw differs from one in
// 64-bit floats only where u is within about 2^-40 of a border.
//
// Most draws need few of a row's logits.  head_kernel looks at the row twice: for the largest of
// each of 1024 slots, and for the logits above a bound, the head, which it sums exactly:
//   top-k       the bound is the k-th largest of the slots, so that at least k are in the head
//   min-p       the least logit that is kept, where nothing else filters
//   otherwise   the 800th largest of the slots; the mass of the rest is summed in fp32, each 8
//               logits' sum a whole number of 2^-42 of the bound's weight
// (rows of up to 2048 logits are all head).  The head is put in buckets of equal width in l, whose
// sums say in which of them a sum of weights crosses its bound, and there few logits are left.
// Then either all that matters lies in the head, clear of what the rest's error could move and of
// how far the two kernels' sums may lie apart, and the draw is what both would say, or the token is
// left as kPending.  order_kernel takes those rows.  A
// logit of 16 bits has one of 65,536 values, and equal logits have equal weights, so the order
// needs no sorting: the numbers of logits of each value say everything.  One pass over the row
// counts them in shared memory (a word for each magnitude, 16 bits a sign, 128 KB); top-k, top-p
// and the draw are then searches in sums over the values in descending order, and a second look at
// the row finds the r-th logit of the value drawn.  Slots and groups of 8 are the row's own: how
// many CTAs share it moves no result.
//
// 32 neighbouring magnitudes are a cell: their steps are equal, so with k steps from its largest
// value, exp(-step / T)^k is the same for all cells of a power of two.  A cell's mass is its first
// value's weight, B, times S = sum of counts times those ratios: one product a value instead of
// one exponential.  Ratios are whole numbers of 2^-44, so S is exact, and a sum up to any logit,
// floor(S * B), grows with it whatever is rounded.
//
// In both a cluster of CTAs shares a row, and its first one decides.
//
// What bounds them.  2048 draws from 32,000 logits: head_kernel 88 us, a quarter of it the fp32 sum
// (13 issue slots a logit of 16 it could take with the exponentials' rate), another the head's
// weights, buckets and searches, the others the two looks and their waits, with four CTAs an SM;
// the 2 % of draws that it leaves 30 us, one round of order_kernel.  That takes 16 to 25 us whatever
// its rows: counting is 5 clocks for 32 logits of an SM (atomics on few words), the rest a chain of
// steps that each wait for the last: settings 1 us, cells 2, their masses 2, sums 2, each search 1 to
// 2, the second look up to 3.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sample.cuh"

namespace hs {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kMags = 32768;            // magnitudes of a 16-bit float
constexpr int kCells = kMags / 32;
constexpr int kRows = 64;               // powers of two with a table of ratios
constexpr int kRowStride = 33;          // (rows a lane apart fall into banks of their own)
constexpr int kMostCtas = 8;
constexpr int kMostVecs = 8191;         // of 8 logits, in a CTA's part: counts fit in 16 bits,
                                        // and a lane has 8 at most
constexpr int32_t kPending = -2;        // the token of a draw that head_kernel leaves ...
constexpr int32_t kClaimed = -3;        // ... and a cluster of order_kernel has taken
constexpr int kOneLog2 = 43;            // a weight of 1: sums of 2^19 stay below 2^63
constexpr int kRatioLog2 = 44;          // a ratio of 1: counts of 2^19 times it too

// ---- values --------------------------------------------------------------------------------
template <bool FP16>
struct Value {
  static constexpr uint32_t kInf = FP16 ? 0x7c00u : 0x7f80u;
  static constexpr int kMant = FP16 ? 10 : 7;
  static constexpr int kRow0 = FP16 ? 0 : 127 - kRows * 3 / 4;  // the first power with a table
  // The bits as a number that grows with the value: -0 is +0, NaN is 0.
  static __device__ __forceinline__ uint32_t key(uint32_t b) {
    const uint32_t mag = b & 0x7fffu;
    uint32_t k = (b & 0x8000u) ? 0xffffu - b : b | 0x8000u;
    if (mag == 0) k = 0x8000u;
    if (mag > kInf) k = 0;
    return k;
  }
  static constexpr uint32_t kLeast = 0xffffu - (0x8000u | kInf);  // minus infinity's: not drawn
  static __device__ __forceinline__ uint32_t bits(uint32_t k) {
    return (k & 0x8000u) ? k & 0x7fffu : 0xffffu - k;
  }
  static __device__ __forceinline__ float number(uint32_t b) {
    if constexpr (FP16) return __half2float(__ushort_as_half((unsigned short)b));
    return __uint_as_float(b << 16);
  }
  // The difference of neighbouring magnitudes at this one.
  static __device__ __forceinline__ float step(uint32_t mag) {
    const uint32_t e = max(mag >> kMant, 1u);
    if constexpr (FP16) return __uint_as_float((e - 25 + 127) << 23);
    return e > 7 ? __uint_as_float((e - 7) << 23) : __uint_as_float(1u << (15 + e));
  }
  // The bits of the least value of the type that is >= x (finite).
  static __device__ __forceinline__ uint32_t bits_from(float x) {
    if constexpr (FP16) return __half_as_ushort(__float2half_ru(x));
    return __bfloat16_as_ushort(__float2bfloat16_ru(x));
  }
  static __device__ __forceinline__ uint32_t ge2(uint32_t a, uint32_t b) {  // 0xffff where a >= b
    if constexpr (FP16)
      return __hge2_mask(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    else
      return __hge2_mask(*reinterpret_cast<const __nv_bfloat162*>(&a),
                         *reinterpret_cast<const __nv_bfloat162*>(&b));
  }
  // 0xffff where a equals b; zeros of both signs do, NaN never.
  static __device__ __forceinline__ uint32_t eq2(uint32_t a, uint32_t b) {
    if constexpr (FP16)
      return __heq2_mask(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    else
      return __heq2_mask(*reinterpret_cast<const __nv_bfloat162*>(&a),
                         *reinterpret_cast<const __nv_bfloat162*>(&b));
  }
  // n + 1 in each half where a >= b; n small.
  static __device__ __forceinline__ uint32_t count_ge2(uint32_t n, uint32_t a, uint32_t b) {
    if constexpr (FP16) {
      const __half2 x = __hadd2(*reinterpret_cast<const __half2*>(&n),
                                __hge2(*reinterpret_cast<const __half2*>(&a),
                                       *reinterpret_cast<const __half2*>(&b)));
      return *reinterpret_cast<const uint32_t*>(&x);
    } else {
      const __nv_bfloat162 x = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&n),
                                       __hge2(*reinterpret_cast<const __nv_bfloat162*>(&a),
                                              *reinterpret_cast<const __nv_bfloat162*>(&b)));
      return *reinterpret_cast<const uint32_t*>(&x);
    }
  }
  static __device__ __forceinline__ float half_of(uint32_t w, int high) {
    if constexpr (FP16) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
      return high ? f.y : f.x;
    }
    return __uint_as_float(high ? w & 0xffff0000u : w << 16);
  }
  static __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {  // NaN loses
    uint32_t r;
    if constexpr (FP16) asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {  // NaN loses
    uint32_t r;
    if constexpr (FP16) asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
};

// ---- weights -------------------------------------------------------------------------------
// 2^(j / 128), j = -64 .. 64, as sums of two floats: exp's series in double, at compile time.
struct Powers {
  float hi[129], lo[129];
  constexpr Powers() : hi(), lo() {
    for (int j = 0; j < 129; ++j) {
      const double x = (j - 64) * 0.69314718055994530942 / 128.0;
      double term = 1.0, sum = 1.0;
      for (int i = 1; i < 24; ++i) {
        term = term * x / i;
        sum += term;
      }
      hi[j] = (float)sum;
      lo[j] = (float)(sum - (double)hi[j]);
    }
  }
};
__device__ const Powers kPowers = Powers();

struct Weight {
  uint64_t w;  // of 2^-44, 2^-1/2 .. 2^1/2; 0 is none
  int32_t n;   // times 2^n, n <= 0
};

// exp((d + dl) / T) for d <= 0, where hi + lo = log2(e) / T.  All steps are on pairs of floats:
// x = d * log2(e) / T, its whole part n, the nearest j / 128 of the rest, and exp of what is left
// (at most 2^-8.5) with its square and higher powers in one float, 2^-18 of the result.
__device__ __forceinline__ Weight weight(float d, float dl, float hi, float lo, const float* p_hi,
                                         const float* p_lo) {
  const float x = __fmul_rn(d, hi);  // (rounded here: its remainder is e)
  Weight r = {0, 0};
  if (!(x >= -62.0f)) return r;      // also where d overflows
  float e = fmaf(d, hi, -x);
  e = fmaf(d, lo, e);
  e = fmaf(dl, hi, e);
  const float n = rintf(x);
  const float f = x - n;                       // exact
  const float j = rintf(f * 128.0f);
  const float z = fmaf(j, -0.0078125f, f);     // exact
  constexpr float kLn2Hi = 0.693147182f, kLn2Lo = -1.90465421e-9f;  // ln 2 as a pair
  const float y = __fmul_rn(z, kLn2Hi);
  float yl = fmaf(z, kLn2Hi, -y);
  yl = fmaf(z, kLn2Lo, yl);
  yl = fmaf(e, kLn2Hi, yl);
  float q = fmaf(y, 0.0416666667f, 0.166666667f);
  q = fmaf(y, q, 0.5f);
  const float pl = fmaf(y * y, q, yl) + y * yl;  // exp - 1 = y + pl
  const int at = (int)j + 64;
  const float th = p_hi[at], tl = p_lo[at];
  const float u = __fmul_rn(th, y);
  const float ul = fmaf(th, y, -u);
  const float s = __fadd_rn(th, u);
  const float t = (th - s) + u;
  const float rest = t + (ul + fmaf(th, pl, fmaf(tl, y, tl)));
  // s is a multiple of 2^-24 below 2
  r.w = ((uint64_t)(uint32_t)(s * 16777216.0f) << 20) +
        (int64_t)__float2int_rn(rest * 17592186044416.0f);
  r.n = (int)n;
  return r;
}

// log2(e) / T as a sum of two floats.
__device__ __forceinline__ void slope(float T, float& hi, float& lo) {
  constexpr float kHi = 1.44269502f, kLo = 1.92596303e-8f;  // log2(e) as a pair
  hi = __fdiv_rn(kHi, T);
  lo = (fmaf(-hi, T, kHi) + kLo) / T;
}

// floor(m * f) for 0 <= f <= 1, exactly; `more` if it is less than m * f.
__device__ __forceinline__ uint64_t part_of(uint64_t m, float f, bool& more) {
  const uint32_t b = __float_as_uint(f), e = b >> 23;
  const uint64_t frac = (b & 0x7fffffu) | (e ? 0x800000u : 0u);
  const int s = 150 - (int)(e ? e : 1u);  // f = frac / 2^s, s >= 23
  const uint64_t lo = m * frac, hi = __umul64hi(m, frac);
  if (s < 64) {
    more = (lo << (64 - s)) != 0;
    return (hi << (64 - s)) | (lo >> s);
  }
  more = lo != 0 || hi != 0;  // (hi < 2^24, and s < 88 leaves some of it)
  if (s >= 88) return 0;
  more = lo != 0 || (s > 64 && (hi << (128 - s)) != 0);
  return hi >> (s - 64);
}

// floor(2^43 * (S / 2^44) * B): grows with S.
__device__ __forceinline__ uint64_t mass_of(uint64_t S, const Weight& B) {
  const uint64_t lo = S * B.w, hi = __umul64hi(S, B.w);
  const int s = 2 * kRatioLog2 - kOneLog2 - B.n;  // 45 .. 107
  return s < 64 ? (hi << (64 - s)) | (lo >> s) : hi >> (s - 64);
}

// ---- a row's part ----------------------------------------------------------------------------
// Logits lie in vectors of 8 that begin at 16-byte boundaries; `off` elements before the row's
// first belong to no row, and are never read.
struct Part {
  const uint16_t* row;
  int32_t off;
  int32_t vocab;
  int32_t v0, v1;  // this CTA's vectors

  __device__ __forceinline__ uint4 load(int32_t v) const {
    const int32_t i = v * 8 - off;
    if (i >= 0 && i + 8 <= vocab) return __ldg(reinterpret_cast<const uint4*>(row + i));
    uint64_t lo = ~0ull, hi = ~0ull;  // NaN: not drawn
#pragma unroll 1
    for (int j = 7; j >= 0; --j) {  // (a loop: this stands in many places)
      const uint64_t b = i + j >= 0 && i + j < vocab ? __ldg(row + i + j) : 0xffffu;
      hi = hi << 16 | lo >> 48;
      lo = lo << 16 | b;
    }
    return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
  }
  // The vectors of a warp: contiguous, so that warps are in the order of the row.
  template <int WARPS>
  __device__ __forceinline__ void warp(int32_t& a, int32_t& b) const {
    const int32_t per = (v1 - v0 + WARPS - 1) / WARPS;
    a = min(v1, v0 + (int32_t)(threadIdx.x >> 5) * per);
    b = min(v1, a + per);
  }
};

__device__ __forceinline__ uint64_t ld_cluster64(uint32_t addr) {
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ void st_cluster(uint32_t addr, uint32_t x) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(x) : "memory");
}

// What another CTA of the cluster holds at the same place, or this one, by a load of its own shared
// memory (the masses of two CTAs' cells 3950 -> 3080 clocks).
__device__ __forceinline__ uint32_t of_cta(const uint32_t* x, uint32_t c, uint32_t rank) {
  return c == rank ? *x : ld_cluster(cluster_smem_addr(x, c));
}
__device__ __forceinline__ uint64_t of_cta(const uint64_t* x, uint32_t c, uint32_t rank) {
  return c == rank ? *x : ld_cluster64(cluster_smem_addr(x, c));
}

// Sums of x over the warp's lanes.
__device__ __forceinline__ uint64_t warp_sum(uint64_t x) {
  // three pieces of 21 bits: 32 of them stay below 2^26
  const uint32_t a = __reduce_add_sync(0xffffffffu, (uint32_t)x & 0x1fffffu);
  const uint32_t b = __reduce_add_sync(0xffffffffu, (uint32_t)(x >> 21) & 0x1fffffu);
  const uint32_t c = __reduce_add_sync(0xffffffffu, (uint32_t)(x >> 42));
  return ((uint64_t)c << 42) + ((uint64_t)b << 21) + a;
}

// A draw's settings, and whether it can be drawn with them.
struct Settings {
  float T, top_p, min_p, u;
  int32_t k, row;
  __device__ __forceinline__ Settings(const SampleParams& p, int32_t i)
      : T(p.temperature ? __ldg(p.temperature + i) : 1.0f),
        top_p(p.top_p ? __ldg(p.top_p + i) : 1.0f),
        min_p(p.min_p ? __ldg(p.min_p + i) : 0.0f),
        u(__ldg(p.u + i)),
        k(p.top_k ? __ldg(p.top_k + i) : 0),
        row(p.row_of ? __ldg(p.row_of + i) : i) {
    if (k < 0 || k >= p.vocab) k = 0;  // all
  }
  __device__ __forceinline__ bool fit(const SampleParams& p) const {
    return (T == 0.0f || (T >= 0x1p-24f && T <= 0x1p24f)) && top_p >= 0.0f && top_p <= 1.0f &&
           min_p >= 0.0f && min_p <= 1.0f && u >= 0.0f && u < 1.0f &&
           (uint32_t)row < (uint32_t)p.n_rows;
  }
};

__device__ __forceinline__ void write_out(const SampleParams& p, int32_t i, int32_t token,
                                          float logprob, uint32_t kept) {
  p.tokens[i] = token;
  if (p.logprob) p.logprob[i] = logprob;
  if (p.kept) p.kept[i] = (int32_t)kept;
}

template <int WARPS>
__device__ __forceinline__ Part part_of_row(const SampleParams& p, int32_t row, uint32_t rank,
                                            uint32_t ctas) {
  Part part;
  part.row = p.logits + (int64_t)row * p.stride;
  part.off = (int32_t)((reinterpret_cast<uintptr_t>(part.row) & 15) / 2);
  part.vocab = p.vocab;
  const int32_t vecs = (p.vocab + part.off + 7) / 8, per = (vecs + (int32_t)ctas - 1) / (int32_t)ctas;
  part.v0 = min(vecs, (int32_t)rank * per);
  part.v1 = min(vecs, part.v0 + per);
  return part;
}

// The least logit that min-p keeps, rounded up.  (Called seldom, and not inlined: its code would be
// fetched with the rest.)
__device__ __noinline__ float least_in_64_bits(float largest, float T, float min_p) {
  return __double2float_ru((double)largest + (double)T * log((double)min_p));
}

// Its bits.  In fp32, unless its error might hold a value of the type.
template <bool FP16>
__device__ __forceinline__ uint32_t least_kept(float largest, float T, float min_p) {
  const float by = T * logf(min_p), least = largest + by;
  const float off = (fabsf(largest) + fabsf(by)) * 0x1p-20f + 0x1p-126f;
  const uint32_t b = Value<FP16>::bits_from(least - off);
  if (b == Value<FP16>::bits_from(fminf(least + off, largest))) return b;
  return Value<FP16>::bits_from(least_in_64_bits(largest, T, min_p));
}

// log of the weight at l over a sum of weights: of two numbers <= 0.  (Not of the token's weight:
// a small one has few bits.)
__device__ __forceinline__ float log_share(float l, float largest, float T, uint64_t mass) {
  const float over = (float)(mass - (1ull << kOneLog2)) * 0x1p-43f;
  return (l == largest ? 0.0f : (l - largest) / T) - log1pf(over);
}

// ---- the head ----------------------------------------------------------------------------------
constexpr int kHeadThreads = 256;  // 4 CTAs an SM: what one waits for, others fill
constexpr int kHeadWarps = kHeadThreads / 32;
constexpr int kHeadEach = 8;                          // logits of a head, a thread
constexpr int kHeadMost = kHeadEach * kHeadThreads;
constexpr int kHeadSlots = 800;   // slots whose largest logits are in a head, for top-k too: of
                                  // 1024, so that about 1024 ln(1024 / 224) = 1560 logits are
                                  // above the bound.  (With 512, 710 logits: 5 us less of the 88
                                  // above, but 11 % of the draws are left, not 2.)
constexpr int kBuckets = 2 * kHeadThreads;
constexpr int kCandidates = kHeadThreads;

// Where a sum crosses a bound.
struct Crossing {
  int32_t bucket;
  uint32_t n;                        // logits of the bucket
  uint32_t count;                    // before it, later with the logit that crosses
  uint64_t mass;
  uint64_t entry;
};

struct HeadShared {
  float hi[129], lo[129];
  uint32_t n, gone, nan;
  int32_t first;
  uint32_t tops[kHeadWarps], counts[kHeadWarps];
  uint64_t rests[kHeadWarps];
  uint64_t rest;
  uint64_t scan_mass[kHeadWarps];
  uint32_t scan_count[kHeadWarps];
  uint32_t own[kHeadThreads], slots[2 * kHeadThreads];  // the largest of even and of odd logits,
                                                        // of this CTA's and of all
  uint32_t mass_lo[kBuckets], mass_hi[kBuckets];
  uint32_t count[kBuckets];
  uint32_t scan_above[kHeadWarps];
  uint64_t ends[2][kHeadWarps];
  Weight edge;
  Crossing crossings[4];
  int32_t candidates[kCandidates];  // places in the list
  uint64_t list[kHeadMost];      // key << 32 | ~index: larger ones come first
  uint64_t weights[kHeadMost];
  uint16_t bucket[kHeadMost];
};

// The largest key that at least k of the slots' are not below, but for its last bit, which is 0.
// Seven candidates at a time, a warp each.
template <bool FP16>
__device__ __forceinline__ uint32_t slots_bound(uint32_t k, HeadShared& sm) {
  using V = Value<FP16>;
  static_assert(kHeadWarps == 8, "a candidate a warp");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t m[kHeadThreads / 16];
#pragma unroll
  for (int j = 0; j < kHeadThreads / 16; ++j) m[j] = sm.slots[j * 32 + lane];
  uint32_t cut = 0;
  for (int shift = 13; shift > 0; shift -= 3) {
    const uint32_t from = V::bits((cut | warp << shift) & 0xffffu) * 0x10001u;
    uint32_t x = 0;
#pragma unroll
    for (int j = 0; j < kHeadThreads / 16; ++j) x = V::count_ge2(x, m[j], from);
    const uint32_t n = __reduce_add_sync(
        0xffffffffu, (uint32_t)(V::number(x & 0xffffu) + V::number(x >> 16)));
    if (shift != 13) __syncthreads();
    if (lane == 0) sm.counts[warp] = n;
    __syncthreads();
    const unsigned enough = __ballot_sync(0xffffffffu, sm.counts[lane % kHeadWarps] >= k) | 1u;
    cut |= (31 - __clz(enough & 0xffu)) << shift;
  }
  return cut;
}

// A CTA's head in buckets of equal width in l, the largest logits first: a thread has two of them,
// with what is before them.  (Searches are rounds of loops here and below: straight code costs a
// short kernel more time to load than to run.)
struct Head {
  HeadShared* sm;
  uint32_t n;
  uint32_t count[2], before;
  uint64_t mass[2], mass_before;

  // An entry's key and place in the row as 35 bits that grow as the order goes.
  static __device__ __forceinline__ uint64_t in_order(uint64_t entry) {
    return (entry >> 32) << 19 | ((uint32_t)entry & 0x7ffffu);
  }
  __device__ __forceinline__ void add(int b, uint64_t w) const {
    const uint32_t part = (uint32_t)w, was = atomicAdd(sm->mass_lo + b, part);
    atomicAdd(sm->mass_hi + b, (uint32_t)(w >> 32) + (was + part < was));
    atomicAdd(sm->count + b, 1u);
  }
  // This thread's buckets and what is before them; returns the sum of all.
  __device__ __forceinline__ uint64_t scan() {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      count[h] = sm->count[2 * tid + h];
      mass[h] = ((uint64_t)sm->mass_hi[2 * tid + h] << 32) + sm->mass_lo[2 * tid + h];
    }
    mass_before = mass[0] + mass[1];
    before = count[0] + count[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, mass_before, o);
      const uint32_t z = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) {
        mass_before += y;
        before += z;
      }
    }
    if (lane == 31) {
      sm->scan_mass[warp] = mass_before;
      sm->scan_count[warp] = before;
    }
    __syncthreads();
    const uint64_t part_mass = lane < kHeadWarps ? sm->scan_mass[lane] : 0;
    const uint32_t part_count = lane < kHeadWarps ? sm->scan_count[lane] : 0;
    mass_before += warp_sum(lane < warp ? part_mass : 0) - mass[0] - mass[1];
    before += __reduce_add_sync(0xffffffffu, lane < warp ? part_count : 0) - count[0] - count[1];
    return warp_sum(part_mass);
  }

  // The first logit with which all up to it have at least `want` of mass and `want_n` are in
  // number (one of them is 0, the other is not).  False if there is none.
  __device__ __forceinline__ bool find(int which, uint64_t want, uint32_t want_n, uint64_t& entry,
                                       uint64_t& upto, uint32_t& number) const {
    const auto reaches = [&](uint64_t m, uint32_t c) { return m >= want && c >= want_n; };
    const int tid = threadIdx.x;
    Crossing& x = sm->crossings[which];
    uint64_t m = mass_before;
    uint32_t k = before;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (reaches(m + mass[h], k + count[h]) && !reaches(m, k)) {
        x.bucket = 2 * tid + h;
        x.mass = m;
        x.count = k;
      }
      m += mass[h];
      k += count[h];
    }
    __syncthreads();
    const int32_t bucket = x.bucket;
    if (bucket < 0) return false;
    uint64_t base = x.mass, low = 0, high = ~0ull;
    uint32_t base_count = x.count;
    const auto chosen = [&](uint32_t s) {
      if (sm->bucket[s] != bucket) return false;
      const uint64_t v = in_order(sm->list[s]);
      return v >= low && v <= high;
    };
    const auto gather = [&](auto&& which) {
      for (uint32_t s = tid; s < n; s += kHeadThreads) {
        if (which(s)) {
          const uint32_t at = atomicAdd(&x.n, 1u);
          if (at < kCandidates) sm->candidates[at] = (int32_t)s;
        }
      }
      __syncthreads();
    };
    gather([&](uint32_t s) { return sm->bucket[s] == bucket; });
    while (x.n > kCandidates) {
      // Too many (equal logits, mostly): in buckets once more, of equal width in the order itself.
      uint64_t least = ~0ull, most = 0;
      for (uint32_t s = tid; s < n; s += kHeadThreads) {
        if (!chosen(s)) continue;
        least = min(least, in_order(sm->list[s]));
        most = max(most, in_order(sm->list[s]));
      }
#pragma unroll 1
      for (int o = 16; o > 0; o /= 2) {
        least = min(least, __shfl_xor_sync(0xffffffffu, least, o));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
      }
      if ((tid & 31) == 0) {
        sm->ends[0][tid >> 5] = least;
        sm->ends[1][tid >> 5] = most;
      }
      for (int j = tid; j < kBuckets; j += kHeadThreads)
        sm->mass_lo[j] = sm->mass_hi[j] = sm->count[j] = 0;
      __syncthreads();
#pragma unroll 1
      for (int w = 0; w < kHeadWarps; ++w) {
        least = min(least, sm->ends[0][w]);
        most = max(most, sm->ends[1][w]);
      }
      const int wide = 64 - __clzll((long long)(most - least)) - 9;
      const int shift = wide > 0 ? wide : 0;
      for (uint32_t s = tid; s < n; s += kHeadThreads)
        if (chosen(s)) add((int)((most - in_order(sm->list[s])) >> shift), sm->weights[s]);
      __syncthreads();
      Head finer;
      finer.sm = sm;
      finer.scan();
      if (tid == 0) x.n = 0;
      m = base + finer.mass_before;
      k = base_count + finer.before;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (reaches(m + finer.mass[h], k + finer.count[h]) && !reaches(m, k)) {
          x.bucket = 2 * tid + h;
          x.mass = m;
          x.count = k;
        }
        m += finer.mass[h];
        k += finer.count[h];
      }
      __syncthreads();
      base = x.mass;
      base_count = x.count;
      high = most - ((uint64_t)x.bucket << shift);
      low = high - ((1ull << shift) - 1);
      gather(chosen);
    }
    // A candidate a thread, each against all.
    const uint32_t c = x.n;
    if (tid < (int)c) {
      const uint64_t v = sm->list[sm->candidates[tid]], w = sm->weights[sm->candidates[tid]];
      uint64_t sum = base;
      uint32_t order = base_count;
      for (uint32_t j = 0; j < c; ++j) {
        const int32_t other = sm->candidates[j];
        if (sm->list[other] > v) {
          sum += sm->weights[other];
          ++order;
        }
      }
      if (reaches(sum + w, order + 1) && !reaches(sum, order)) {
        x.entry = v;
        x.mass = sum + w;  // (nobody reads the base any more)
        x.count = order + 1;
      }
    }
    __syncthreads();
    entry = x.entry;
    upto = x.mass;
    number = x.count;
    return true;
  }
};

template <bool FP16>
__global__ void __launch_bounds__(kHeadThreads, 4) head_kernel(const SampleParams p) {
  __shared__ HeadShared sm;
  using V = Value<FP16>;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t ctas;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
  const uint32_t rank = cluster_ctarank();
  const int32_t i = blockIdx.x / ctas;
  if (tid < 129) {
    sm.hi[tid] = kPowers.hi[tid];
    sm.lo[tid] = kPowers.lo[tid];
  }
  for (int j = tid; j < kBuckets; j += kHeadThreads) sm.mass_lo[j] = sm.mass_hi[j] = sm.count[j] = 0;
  if (tid == 0) {
    sm.n = sm.gone = sm.nan = 0;
    sm.first = 0x7fffffff;
  }
  if (tid < 4) {
    sm.crossings[tid].bucket = -1;
    sm.crossings[tid].n = 0;
  }
  pdl_wait();
  pdl_trigger();
  const int32_t live = p.n_dev ? __ldg(p.n_dev) : p.n;
  const Settings set(p, i);
  if (i >= live) return;
  const bool lead = rank == 0 && tid == 0;
  if (!set.fit(p)) {
    if (lead) {
      write_out(p, i, -1, -INFINITY, 0);
      set_error(p.err, kErrInvalidArg);
    }
    return;
  }
  // Vectors of 8 logits: CTA c takes c, c + ctas, ... of each 256, a thread one of them.  A slot
  // is the even or the odd logits of all vectors that are 512 apart.
  const Part part = part_of_row<kHeadWarps>(p, set.row, 0, 1);
  const int32_t vecs = part.v1, stride = kHeadThreads * (int32_t)ctas;
  const int32_t steps = (vecs + 8 * stride - 1) / (8 * stride);
  const int32_t v_first = tid + kHeadThreads * (int32_t)rank;

  // ---- the largest ---------------------------------------------------------------------------
  uint32_t best[2] = {(0x8000u | V::kInf) * 0x10001u, (0x8000u | V::kInf) * 0x10001u}, mags = 0;
  uint4 x[8];  // of the last step: what most rows need no second load for
  for (int32_t s = 0; s < steps; ++s) {
    const int32_t v = v_first + s * 8 * stride;
#pragma unroll
    for (int h = 0; h < 8; ++h)
      if (v + h * stride < vecs) x[h] = part.load(v + h * stride);
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      if (v + h * stride >= vecs) break;
      const uint32_t w[4] = {x[h].x, x[h].y, x[h].z, x[h].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        best[h & 1] = V::max2(best[h & 1], w[j]);
        asm("max.u16x2 %0, %0, %1;" : "+r"(mags) : "r"(w[j] & 0x7fff7fffu));
      }
    }
  }
  const bool odd = max(mags & 0xffffu, mags >> 16) >= V::kInf;  // NaN or infinities among them
  if (ctas > 1) {
    // (an even or an odd CTA's vectors)
    best[0] = V::max2(best[0], best[1]);
    sm.own[tid] = best[0];
    cluster_sync();
    uint32_t others[kMostCtas];
#pragma unroll
    for (uint32_t c = 0; c < kMostCtas; ++c)
      others[c] = ld_cluster(cluster_smem_addr(sm.own + tid, c < ctas ? c : c & 1));
#pragma unroll
    for (int h = 0; h < 2; ++h)
      best[h] = V::max2(V::max2(others[h], others[h + 2]), V::max2(others[h + 4], others[h + 6]));
  }
  sm.slots[tid] = best[0];
  sm.slots[kHeadThreads + tid] = best[1];
  const uint32_t both = V::max2(best[0], best[1]);
  const uint32_t warp_top =
      __reduce_max_sync(0xffffffffu, max(V::key(both & 0xffffu), V::key(both >> 16)));
  if (lane == 0) sm.tops[warp] = warp_top;
  __syncthreads();
  const uint32_t top = __reduce_max_sync(0xffffffffu, sm.tops[lane % kHeadWarps]);
  const uint32_t top_bits = V::bits(top);
  const bool infinite = top_bits == V::kInf;
  if (top <= V::kLeast ||
      (set.T != 0.0f && !p.whole && (infinite || set.k > kHeadSlots))) {
    if (lead) {
      if (top <= V::kLeast) write_out(p, i, -1, -INFINITY, 0);
      else p.tokens[i] = kPending;
    }
    if (ctas > 1) cluster_sync();  // nobody leaves while it is read
    return;
  }
  const float largest = V::number(top_bits);

  // ---- its place, or the head's bound ----------------------------------------------------------
  if (set.T == 0.0f) {
    const uint32_t twice = top_bits * 0x10001u;
    int32_t first = 0x7fffffff;
    for (int32_t s = 0; s < steps && first == 0x7fffffff; ++s) {
      const int32_t v = v_first + s * 8 * stride;
      if (steps > 1) {
#pragma unroll
        for (int h = 0; h < 8; ++h)
          if (v + h * stride < vecs) x[h] = part.load(v + h * stride);
      }
#pragma unroll
      for (int h = 0; h < 8; ++h) {
        if (v + h * stride >= vecs || first != 0x7fffffff) break;
        const uint32_t w[4] = {V::eq2(x[h].x, twice), V::eq2(x[h].y, twice), V::eq2(x[h].z, twice),
                               V::eq2(x[h].w, twice)};
#pragma unroll
        for (int j = 3; j >= 0; --j)
          if (w[j]) first = (v + h * stride) * 8 + 2 * j + ((w[j] & 1u) ? 0 : 1) - part.off;
      }
    }
    first = __reduce_min_sync(0xffffffffu, first);
    if (lane == 0 && first != 0x7fffffff) atomicMin(&sm.first, first);
    if (ctas > 1) cluster_sync(); else __syncthreads();
    if (lead) {
      for (uint32_t c = 0; c < ctas; ++c)
        first = min(first, (int32_t)ld_cluster(cluster_smem_addr(&sm.first, c)));
      write_out(p, i, first, 0.0f, 1);
    }
    if (ctas > 1) cluster_sync();
    return;
  }
  const bool by_k = set.k > 0;
  const bool by_min = !p.whole && !by_k && set.top_p >= 1.0f && set.min_p > 0.0f;
  const bool with_rest = !p.whole && !by_k && !by_min;
  const uint32_t least_bits = set.min_p > 0.0f && !infinite
                                  ? least_kept<FP16>(largest, set.T, set.min_p)
                                  : 0x8000u | (V::kInf - 1);
  // The key of the head's least logit.
  uint32_t cut = 0;
  if (infinite) cut = top;  // (beside which nothing has weight)
  else if (by_min) cut = V::key(least_bits);
  else if (!p.whole) cut = slots_bound<FP16>(by_k ? set.k : kHeadSlots, sm);
  cut = max(cut, V::kLeast + 1);
  float c_hi, c_lo;
  slope(set.T, c_hi, c_lo);
  // What has no weight at all, as logits that a mask holds at the type's lowest value, is in no head
  // (but in one of a whole row, which has to decide all).
  if (!p.whole && !by_min)
    cut = max(cut, V::key(V::bits_from(largest - __fdiv_rn(64.0f, c_hi))));
  const uint32_t cut_bits = V::bits(cut);
  const float edge = V::number(cut_bits);

  // ---- the head, and the rest's mass -----------------------------------------------------------
  // Of each value 2^((l - edge) log2(e) / T), 1 where that is more, so that logits of the head
  // count 1 (and NaN too): they are taken off in the end.  A value is right to 2^-22 by ex2, and
  // to 3 * 2^-24 ln 2 times its exponent, by the roundings of l - edge, of the slope and of their
  // product: to 2^-17 in all up to an exponent of 50, and below that it is less than the last place
  // of the sums.  Sums of 8 add 3 * 2^-24; they become whole numbers of 2^-42 in two pieces.
  uint32_t sum_hi = 0, gone = 0, nan = 0;
  int32_t sum_lo = 0;
  const uint32_t cut2 = cut_bits * 0x10001u;
  for (int32_t s = steps - 1; s >= 0; --s) {
    const int32_t v = v_first + s * 8 * stride;
    if (s != steps - 1) {
#pragma unroll
      for (int h = 0; h < 8; ++h) x[h] = part.load(v + h * stride);
    }
    uint32_t hits[2] = {0, 0};  // of 4 vectors each, even logits in the low half
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      if (v + h * stride >= vecs) break;
      const uint32_t w[4] = {x[h].x, x[h].y, x[h].z, x[h].w};
      uint32_t in = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) in |= V::ge2(w[j], cut2) & (0x00010001u << j);
      hits[h / 4] |= in << (4 * (h % 4));
      if (with_rest) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t near = V::min2(w[j], cut2);
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const float d = __fadd_rn(V::half_of(near, q), -edge);
            asm("ex2.approx.ftz.f32 %0, %1;"
                : "=f"(e[2 * j + q])
                : "f"(__fmul_rn(d, c_hi)));
          }
        }
        const float sum = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        // (at most 8; places of 2^-19 at 24, of 2^-42 at 1.5 * 2^-19)
        constexpr float kAt = 24.0f, kBelow = 0x1.8p-19f;
        const float t = __fadd_rn(sum, kAt);
        const float u = __fadd_rn(__fadd_rn(sum, -__fadd_rn(t, -kAt)), kBelow);
        sum_hi += __float_as_uint(t) - __float_as_uint(kAt);
        sum_lo += (int32_t)(__float_as_uint(u) - __float_as_uint(kBelow));
      }
      if (odd && !by_min) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t a = w[j] & 0x7fff7fffu;
          gone += __popc(__vcmpgeu2(a, V::kInf * 0x10001u)) / 16;
          nan += __popc(__vcmpgtu2(a, V::kInf * 0x10001u)) / 16;
        }
      }
    }
    if (hits[0] | hits[1]) {
      uint32_t at = atomicAdd(&sm.n, __popc(hits[0]) + __popc(hits[1]));
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        for (uint32_t m = hits[g]; m; m &= m - 1, ++at) {
          const int bit = __ffs(m) - 1;
          const int32_t h = g * 4 + (bit & 15) / 4;
          const int32_t l = (v + h * stride) * 8 + 2 * (bit & 3) + (bit >> 4) - part.off;
          if (at < kHeadMost)
            sm.list[at] = (uint64_t)V::key(__ldg(part.row + l)) << 32 | ~(uint32_t)l;
        }
      }
    }
  }
  gone = __reduce_add_sync(0xffffffffu, gone);
  if (lane == 0 && gone) atomicAdd(&sm.gone, gone);
  if (with_rest) {
    const uint64_t S = warp_sum(((uint64_t)sum_hi << (kRatioLog2 - 19)) + (int64_t)sum_lo * 4);
    nan = __reduce_add_sync(0xffffffffu, nan);
    if (lane == 0) {
      sm.rests[warp] = S;
      if (nan) atomicAdd(&sm.nan, nan);
    }
    __syncthreads();
    if (warp == 0) {
      const uint64_t all = warp_sum(lane < kHeadWarps ? sm.rests[lane] : 0);
      if (lane == 0) sm.rest = all - ((uint64_t)(sm.n + sm.nan) << kRatioLog2);
    }
  }
  if (ctas > 1) cluster_sync(); else __syncthreads();
  if (rank == 0) {
    // All CTAs' lists behind this one's, a few warps for each.
    const bool has = lane < (int)ctas;
    const uint32_t theirs = has ? ld_cluster(cluster_smem_addr(&sm.n, lane)) : 0;
    const uint32_t n = __reduce_add_sync(0xffffffffu, theirs);
    gone = __reduce_add_sync(0xffffffffu, has ? ld_cluster(cluster_smem_addr(&sm.gone, lane)) : 0);
    uint64_t S = 0;
    if (with_rest) {
      uint64_t r = has ? ld_cluster64(cluster_smem_addr(&sm.rest, lane)) : 0;
#pragma unroll
      for (int o = 1; o < kMostCtas; o <<= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
      S = __shfl_sync(0xffffffffu, r, 0);
      if ((int64_t)S < 0) S = 0;  // (by its rounding)
    }
    if (n > kHeadMost) {
      if (tid == 0) p.tokens[i] = kPending;
    } else {
      const int c = warp % ctas;  // (8 CTAs at most)
      if (c > 0) {
        const uint32_t at = __reduce_add_sync(0xffffffffu, lane < c ? theirs : 0);
        const uint32_t number = __shfl_sync(0xffffffffu, theirs, c);
        for (uint32_t j = warp / ctas * 32 + lane; j < number; j += kHeadWarps / ctas * 32)
          sm.list[at + j] = ld_cluster64(cluster_smem_addr(sm.list + j, c));
      }
      __syncthreads();
      // Weights, and their sums in buckets.
      Head head;
      head.sm = &sm;
      head.n = n;
      const float range = fminf(largest - edge, __fdiv_rn(62.0f, c_hi));
      const float scale = range > 0.0f ? fminf(__fdiv_rn((float)kBuckets, range), 1e30f) : 0.0f;
      const uint32_t least_key = V::key(least_bits);
      uint32_t above = 0;  // that min-p keeps
#pragma unroll 1
      for (uint32_t s = tid; s < n + with_rest; s += kHeadThreads) {  // (the last is the bound)
        const uint32_t key = s < n ? (uint32_t)(sm.list[s] >> 32) : cut;
        const float l = V::number(V::bits(key));
        const float d = key == top ? 0.0f : l - largest, bb = d - l;
        const float dl = key == top ? 0.0f : (l - (d - bb)) - (largest + bb);
        const Weight x = weight(d, dl, c_hi, c_lo, sm.hi, sm.lo);
        if (s == n) {
          sm.edge = x;
          break;
        }
        const int shift = kRatioLog2 - kOneLog2 - x.n;
        const uint64_t w = (x.w + (1ull << (shift - 1))) >> shift;
        const int32_t b = min((int32_t)(-d * scale), kBuckets - 1);
        sm.weights[s] = w;
        sm.bucket[s] = (uint16_t)b;
        above += key >= least_key;
        head.add(b, w);
      }
      above = __reduce_add_sync(0xffffffffu, above);
      if (lane == 0) sm.scan_above[warp] = above;
      __syncthreads();
      const uint64_t all_mass = head.scan();
      above = __reduce_add_sync(0xffffffffu, lane < kHeadWarps ? sm.scan_above[lane] : 0);

      // What is kept and its mass, uncertain by `off`: by the rest's error, and where order_kernel
      // might be asked instead by how far its sum may lie from this one, so that a draw is decided
      // here only if it would be decided so there: two sums of `kept` logits, each right to 2^-41 of
      // itself and 1 for each logit, and any two of fewer logits.
      // (what is gone counts what a vector has beside the row)
      const uint32_t all = (p.vocab + part.off + 7) / 8 * 8 - gone;
      uint32_t kept = by_k ? min((uint32_t)set.k, infinite ? n : all) : with_rest ? all : n;
      uint64_t mass = all_mass, entry = 0;
      const auto apart = [&]() { return p.either ? (mass >> 40) + 2 * (uint64_t)kept + 2 : 0; };
      uint64_t off = 0;
      if (with_rest && kept > n) {
        // Its error: 2^-17 of it, and 2^-20 of the 1 that each of the others counted.
        mass += mass_of(S, sm.edge);
        off = mass_of((S >> 17) + ((uint64_t)(n + gone) << (kRatioLog2 - 20)), sm.edge) + 2;
      }
      uint64_t between = apart();
      off += between;
      bool clear = true;
#pragma unroll 1
      for (int step = 0; step < 4 && clear; ++step) {  // top-k, top-p, min-p, the draw
        uint64_t want = 0, most = 0, upto_it;
        uint32_t want_n = 0, number_of_it;
        if (step == 0) {
          if (!by_k || n <= (uint32_t)set.k) continue;
          want_n = set.k;
        } else if (step == 2) {
          if (!(set.min_p > 0.0f) || above >= kept) continue;
          if (above == n && least_key < cut) {  // it might keep some of the rest
            clear = false;
            break;
          }
          want_n = above;
        } else {
          const float share = step == 1 ? set.top_p : set.u;
          if (step == 1 && !(share < 1.0f)) continue;
          bool more;
          want = part_of(mass - off, share, more);
          want += more || step == 3;  // (of a draw's sum, more than that)
          want = want > between ? want - between : 1;
          most = part_of(mass + off, share, more);
          most = max((uint64_t)1, most + (more || step == 3)) + between;
        }
        clear = head.find(step, want, want_n, entry, upto_it, number_of_it) && upto_it >= most;
        if (step < 3) {
          mass = upto_it;
          kept = number_of_it;
          off = between = apart();
        }
      }
      if (tid == 0) {
        if (clear) {
          const float l = V::number(V::bits((uint32_t)(entry >> 32)));
          write_out(p, i, (int32_t)~(uint32_t)entry, log_share(l, largest, set.T, mass), kept);
        } else {
          p.tokens[i] = kPending;
        }
      }
    }
  }
  if (ctas > 1) cluster_sync();  // nobody leaves while it is read
}

// ---- the whole order ---------------------------------------------------------------------------
// Entry e of the order: cells of positive values downwards, then of negative ones.
constexpr int kEntries = 2 * kCells;

struct Shared {
  float hi[129], lo[129];
  // The draw, for all of the CTA: what lies here is not held in registers from barrier to barrier,
  // and so is not among what is spilled (a cluster's barrier sends that to the second-level cache:
  // 192 bytes a thread are still stored and loaded in bf16, 144 and 136 in fp16).
  struct {
    float T, top_p, min_p, u;
    int32_t k;
    float c_hi, c_lo;  // log2(e) / T
    uint32_t best;     // bits of the largest logit
    uint32_t ctas;
    Part part;
  } draw;
  // a CTA's own
  int32_t next;                  // the draw to do next
  int32_t pending;               // how far on in the walk the next one that is left stands
  uint32_t top;                  // its largest key
  uint32_t found;                // the bits of the value to find here, 0xffff: none
  uint32_t found_rank;           // how many of it come before
  uint32_t keys[kWarps];
  int32_t hits[kWarps];
  uint32_t n_cells;              // cells with logits, and which
  uint16_t cells[kCells];
  uint64_t scan_mass[kWarps];
  uint32_t scan_count[kWarps];
  uint64_t ratio[kRows * kRowStride];
  // S and the number of logits of each entry; in the leading CTA then the sums of all before it
  uint64_t mass[kEntries + 2];
  uint32_t count[kEntries + 2];
  // of this CTA's share of the entries: the row's mass and number of each, and the weight of its
  // first value (w << 6 | -n); in the leading CTA also both sums up to each 64 entries' end
  uint64_t all_mass[kEntries];
  uint32_t all_count[kEntries];
  uint64_t all_first[kEntries];
  uint64_t upto_mass[kWarps];
  uint32_t upto_count[kWarps];
};

// What a search in the order says: a logit of which value, and the sums up to it.
struct Place {
  uint32_t at;      // entry * 32 + lane
  uint32_t before;  // logits of the value that come before it
  uint32_t count;   // up to it, with it
  uint64_t mass;
};

// Where the count of a magnitude lies: 32 lanes that read one of each of 32 cells, or 32 of one
// cell, read 32 banks.
__device__ __forceinline__ uint32_t place_of(uint32_t mag) { return mag ^ ((mag >> 5) & 31u); }

template <bool FP16>
struct Order {
  using V = Value<FP16>;
  Shared* sm;
  const uint32_t* hist;

  // Where a cell's values begin: its largest, or the row's.
  __device__ __forceinline__ uint32_t head(uint32_t cell, bool neg) const {
    const uint32_t top = sm->draw.best, mag = top & 0x7fffu;
    if (neg) return (top & 0x8000u) ? max(cell * 32, mag) : cell * 32;
    return min(cell * 32 + 31, mag);
  }
  // That value's weight.
  __device__ __forceinline__ Weight first(uint32_t cell, bool neg) const {
    const float t = V::number(sm->draw.best);
    const float l = V::number(head(cell, neg) | (neg ? 0x8000u : 0u));
    const float d = l - t, bb = d - l;
    return weight(d, (l - (d - bb)) - (t + bb), sm->draw.c_hi, sm->draw.c_lo, sm->hi, sm->lo);
  }
  // exp(-k * step / T), in units of 2^-44.
  __device__ __forceinline__ uint64_t ratio(uint32_t mag, int k) const {
    const Weight r = weight(-k * V::step(mag), 0.0f, sm->draw.c_hi, sm->draw.c_lo, sm->hi, sm->lo);
    return r.w >> -r.n;
  }
  __device__ __forceinline__ uint64_t ratio_of(uint32_t cell, int k) const {
    const uint32_t row = (cell * 32 >> V::kMant) - V::kRow0;
    return row < kRows ? sm->ratio[row * kRowStride + k] : ratio(cell * 32, k);
  }
  // How many logits there are with a magnitude, of both signs, from a word of counts.
  static __device__ __forceinline__ void split(uint32_t mag, uint32_t w, uint32_t& pos,
                                               uint32_t& neg) {
    pos = w & 0xffffu;
    neg = w >> 16;
    if (mag == 0) {
      pos += neg;
      neg = 0;
    }
    if (mag > V::kInf) pos = 0;
    if (mag >= V::kInf) neg = 0;
  }
  // ... in all of the row, for the leading CTA.
  __device__ __forceinline__ void counted(uint32_t mag, uint32_t& pos, uint32_t& neg) const {
    const uint32_t ctas = sm->draw.ctas;
    uint32_t w[kMostCtas];
#pragma unroll
    for (uint32_t c = 0; c < kMostCtas; ++c)
      if (c < ctas) w[c] = of_cta(hist + place_of(mag), c, 0);
    pos = neg = 0;
#pragma unroll
    for (uint32_t c = 0; c < kMostCtas; ++c) {
      if (c < ctas) {
        uint32_t x, y;
        split(mag, w[c], x, y);
        pos += x;
        neg += y;
      }
    }
  }
  // S and the number of logits of this CTA's part in each cell, both signs.  Logits lie in few
  // powers of two: the cells that have any are listed first, a thread looking at one, and then
  // summed, four threads each and sign.
  __device__ __forceinline__ void cell_sums() const {
    const uint32_t tid = threadIdx.x, lane = tid & 31;
    uint32_t any = 0;
#pragma unroll
    for (uint32_t k = 0; k < 32; ++k) any |= hist[tid * 32 + (k ^ lane)];
    sm->mass[kCells - 1 - tid] = sm->mass[kCells + tid] = 0;
    sm->count[kCells - 1 - tid] = sm->count[kCells + tid] = 0;
    const unsigned m = __ballot_sync(0xffffffffu, any != 0 && tid * 32 < V::kInf);
    uint32_t at = 0;
    if (lane == 0 && m) at = atomicAdd(&sm->n_cells, __popc(m));
    at = __shfl_sync(0xffffffffu, at, 0) + __popc(m & lanemask_lt());
    if (m >> lane & 1u) sm->cells[at] = (uint16_t)tid;
    __syncthreads();
    const uint32_t n = sm->n_cells;
#pragma unroll 1
    for (uint32_t i0 = tid - lane; i0 < 8 * n; i0 += kThreads) {  // four lanes each, 8 values a lane
      const uint32_t i = (i0 + lane) / 4, k0 = (lane & 3) * 8;
      const bool on = i < 2 * n, neg = on && i >= n;
      const uint32_t cell = sm->cells[on ? neg ? i - n : i : 0], in = cell & 31;
      const uint32_t row = (cell * 32 >> V::kMant) - V::kRow0;
      const uint64_t* r = sm->ratio + min(row, (uint32_t)kRows - 1) * kRowStride;
      // magnitudes downwards for positive values, upwards for negative ones; the row's largest may
      // be further on than the first
      const uint32_t flip = neg ? in : in ^ 31u, shift = neg ? 16 : 0;
      const int skip = neg ? (int)(head(cell, true) - cell * 32) : (int)(cell * 32 + 31 - head(cell, false));
      uint64_t S = 0;
      uint32_t number = 0;
#pragma unroll
      for (uint32_t k = k0; k < k0 + 8; ++k) {
        uint32_t c = hist[cell * 32 + (k ^ flip)] >> shift & 0xffffu;
        if (cell == 0 && k == (neg ? 0u : 31u)) c = neg ? 0 : c + (hist[0] >> 16);  // -0 is 0
        number += c;
        S += c * r[max((int)k - skip, 0)];
      }
      if (number && row >= (uint32_t)kRows) {  // (not in the table)
        S = 0;
#pragma unroll 1
        for (uint32_t k = k0; k < k0 + 8; ++k) {
          uint32_t c = hist[cell * 32 + (k ^ flip)] >> shift & 0xffffu;
          if (cell == 0 && k == (neg ? 0u : 31u)) c = neg ? 0 : c + (hist[0] >> 16);
          if (c) S += c * ratio(cell * 32, (int)k - skip);
        }
      }
#pragma unroll
      for (int o = 1; o < 4; o *= 2) {
        S += __shfl_xor_sync(0xffffffffu, S, o);
        number += __shfl_xor_sync(0xffffffffu, number, o);
      }
      const uint32_t e = neg ? kCells + cell : kCells - 1 - cell;
      if (on && k0 == 0) {
        sm->mass[e] = S;
        sm->count[e] = number;
      }
    }
  }

  // The following by a whole warp.
  // An entry's 32 values, one a lane: how many, and the sums of count * ratio before.
  struct Values {
    uint32_t n, before;
    uint64_t r, S;
    Weight B;
  };
  __device__ __forceinline__ Values values(uint32_t e) const {
    const int lane = threadIdx.x & 31;
    const bool neg = e >= kCells;
    const uint32_t cell = neg ? e - kCells : kCells - 1 - e;
    const uint32_t h = head(cell, neg), mag = neg ? h + lane : h - lane;
    Values v = {};
    if (mag / 32 == cell) {
      uint32_t p, m;
      counted(mag, p, m);
      v.n = neg ? m : p;
    }
    v.r = ratio_of(cell, lane);
    const uint32_t share = kEntries / sm->draw.ctas, whose = e / share;
    const uint64_t packed = of_cta(sm->all_first + (e - whose * share), whose, 0);
    v.B = {packed >> 6, -(int32_t)(packed & 63u)};
    uint32_t c = v.n;
    uint64_t s = v.n * v.r;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t cc = __shfl_up_sync(0xffffffffu, c, o);
      const uint64_t ss = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) {
        c += cc;
        s += ss;
      }
    }
    v.before = c - v.n;
    v.S = s - v.n * v.r;
    return v;
  }
  // From one lane to all.
  __device__ __forceinline__ Place place(bool mine, uint32_t e, uint32_t before, uint32_t count,
                                         uint64_t mass) const {
    const unsigned m = __ballot_sync(0xffffffffu, mine);
    const int from = m ? __ffs(m) - 1 : 31;
    return {e * 32 + from, __shfl_sync(0xffffffffu, before, from),
            __shfl_sync(0xffffffffu, count, from), __shfl_sync(0xffffffffu, mass, from)};
  }
  // The first logit with which all up to it have at least `want` of mass and `want_n` are in
  // number (one of them is 0, the other is not; both are at most all of the row's).  Or, of `value`
  // (bits, not above the largest's), the last logit of that value, or what is before it.
  __device__ __forceinline__ Place find(uint64_t want, uint32_t want_n, int32_t value) const {
    const int lane = threadIdx.x & 31;
    uint32_t e = 0, which = 0;
    if (value >= 0) {
      const bool neg = value > 0x8000;
      const uint32_t mag = value & 0x7fff, cell = mag / 32, h = head(cell, neg);
      e = neg ? kCells + cell : kCells - 1 - cell;
      which = neg ? mag - h : h - mag;
    } else {
      // Which 64 entries, then which of them: two a lane.
      static_assert(kEntries == 64 * kWarps, "two entries a thread");
      unsigned m = __ballot_sync(0xffffffffu,
                                 sm->upto_count[lane] >= want_n && sm->upto_mass[lane] >= want);
      e = (m ? __ffs(m) - 1 : kWarps - 1) * 64;
      const uint32_t at = e + 2 * lane + 1;
      const unsigned odd = __ballot_sync(0xffffffffu, sm->count[at] >= want_n && sm->mass[at] >= want);
      m = __ballot_sync(0xffffffffu, sm->count[at + 1] >= want_n && sm->mass[at + 1] >= want);
      const int l = m ? __ffs(m) - 1 : 31;
      e += 2 * l + !(odd >> l & 1u);
    }
    const Values v = values(e);
    const uint64_t base = sm->mass[e];
    const uint32_t before = sm->count[e] + v.before;
    // With lo logits of the value the bound is not reached, with hi it is.
    uint32_t lo = 0, hi = v.n;
    bool mine = lane == (int)which;
    uint64_t upto = base + mass_of(v.S + hi * v.r, v.B);
    if (value < 0) {
      mine = v.n > 0 && before + hi >= want_n && upto >= want;
      uint64_t sum = base + mass_of(v.S, v.B);
      mine = mine && !(before >= want_n && sum >= want);
#pragma unroll 1
      while (mine && hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        sum = base + mass_of(v.S + mid * v.r, v.B);
        if (before + mid >= want_n && sum >= want) {
          hi = mid;
          upto = sum;
        } else {
          lo = mid;
        }
      }
    }
    return place(mine, e, hi - 1, before + hi, upto);
  }
  __device__ __forceinline__ uint32_t bits_at(uint32_t at) const {
    const uint32_t e = at / 32, lane = at % 32;
    if (e >= kCells) return 0x8000u | (head(e - kCells, true) + lane);
    return head(kCells - 1 - e, false) - lane;
  }
};

// Notes where the logit stands that a draw has found, by the CTA whose part has it.  (A function of
// its own: inlined, it would have the steps before it spill registers.)
template <bool FP16>
__device__ __noinline__ void find_place(int32_t* token, Shared& sm) {
  using V = Value<FP16>;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t twice = sm.found * 0x10001u;
  const Part part = sm.draw.part;
  int32_t a, b;
  part.warp<kWarps>(a, b);
  uint64_t hits = 0;  // a byte for each of this lane's vectors, 8 at most
#pragma unroll 1
  for (int s = 0; s < 8; s += 4) {
    const int32_t v = a + lane + 32 * s;
    uint4 x[4];
#pragma unroll
    for (int h = 0; h < 4; ++h)
      if (v + 32 * h < b) x[h] = part.load(v + 32 * h);
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      if (v + 32 * h >= b) break;
      const uint32_t w[4] = {V::eq2(x[h].x, twice), V::eq2(x[h].y, twice), V::eq2(x[h].z, twice),
                             V::eq2(x[h].w, twice)};
      if (w[0] | w[1] | w[2] | w[3]) {
        uint32_t byte = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) byte |= (w[j] & 1u) << (2 * j) | (w[j] >> 31) << (2 * j + 1);
        hits |= (uint64_t)byte << (8 * (s + h));
      }
    }
  }
  const int32_t mine = (int32_t)__reduce_add_sync(0xffffffffu, __popcll(hits));
  if (lane == 0) sm.hits[warp] = mine;
  __syncthreads();
  int32_t left = (int32_t)sm.found_rank -
                 (int32_t)__reduce_add_sync(0xffffffffu, lane < warp ? sm.hits[lane] : 0);
  if (left < 0 || left >= mine) return;
#pragma unroll 1
  for (int32_t v0 = a; v0 < b; v0 += 32, hits >>= 8) {
    uint32_t byte = (uint32_t)hits & 0xffu;
    const int32_t c = __popc(byte), all = (int32_t)__reduce_add_sync(0xffffffffu, (uint32_t)c);
    if (left >= all) {
      left -= all;
      continue;
    }
    int32_t upto = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t t = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += t;
    }
    if (left >= upto - c && left < upto) {
      for (int32_t skip = left - (upto - c); skip; --skip) byte &= byte - 1;
      *token = (v0 + lane) * 8 + __ffs(byte) - 1 - part.off;
    }
    return;
  }
}

// One draw, by a cluster.
template <bool FP16>
__device__ __forceinline__ void draw_row(const SampleParams& p, int32_t i, uint32_t* hist, Shared& sm,
                                         uint4* zeroed) {
  using V = Value<FP16>;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_ctarank();
  const Settings set(p, i);
  if (!set.fit(p)) {
    if (rank == 0 && tid == 0) {
      write_out(p, i, -1, -INFINITY, 0);
      set_error(p.err, kErrInvalidArg);
    }
    return;
  }
  __syncthreads();  // (some warps may still be at the draw before)
  for (int j = tid; j < kMags / 4; j += kThreads) zeroed[j] = make_uint4(0, 0, 0, 0);
  if (tid == 0) {
    sm.found = 0xffffu;
    sm.n_cells = 0;
    sm.draw.T = set.T;
    sm.draw.top_p = set.top_p;
    sm.draw.min_p = set.min_p;
    sm.draw.u = set.u;
    sm.draw.k = set.k;
    slope(set.T, sm.draw.c_hi, sm.draw.c_lo);
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(sm.draw.ctas));
    sm.draw.part = part_of_row<kWarps>(p, set.row, rank, sm.draw.ctas);
  }
  __syncthreads();

  // ---- count -------------------------------------------------------------------------------
  const Order<FP16> order{&sm, hist};
  // The ratios of the powers of two that logits have (others are few, and taken one by one).
  for (int r = warp; r < (FP16 ? 32 : kRows); r += kWarps)
    sm.ratio[r * kRowStride + lane] = order.ratio((uint32_t)(V::kRow0 + r) << V::kMant, lane);
  uint32_t seen = (0x8000u | V::kInf) * 0x10001u;
  Part part = sm.draw.part;
  int32_t a, b;
  part.warp<kWarps>(a, b);
  for (int32_t v = a + lane; v < b; v += 128) {
    uint4 x[4];
#pragma unroll
    for (int h = 0; h < 4; ++h)
      if (v + 32 * h < b) x[h] = part.load(v + 32 * h);
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      if (v + 32 * h >= b) break;
      const uint32_t w[4] = {x[h].x, x[h].y, x[h].z, x[h].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        seen = V::max2(seen, w[j]);
        atomicAdd(hist + place_of(w[j] & 0x7fffu), (w[j] & 0x8000u) ? 0x10000u : 1u);
        atomicAdd(hist + place_of(w[j] >> 16 & 0x7fffu), (int32_t)w[j] < 0 ? 0x10000u : 1u);
      }
    }
  }
  uint32_t most = __reduce_max_sync(0xffffffffu, max(V::key(seen & 0xffffu), V::key(seen >> 16)));
  if (lane == 0) sm.keys[warp] = most;
  __syncthreads();
  most = __reduce_max_sync(0xffffffffu, sm.keys[lane]);
  if (tid == 0) sm.top = most;
  cluster_sync();
  if (warp == 0) {
    most = lane < sm.draw.ctas ? ld_cluster(cluster_smem_addr(&sm.top, lane)) : 0;
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) sm.draw.best = most <= V::kLeast ? 0xffffffffu : V::bits(most);
  }
  __syncthreads();
  if (sm.draw.best == 0xffffffffu) {
    if (rank == 0 && tid == 0) write_out(p, i, -1, -INFINITY, 0);
    cluster_sync();  // (the next draw writes what others still read)
    return;
  }
  const bool infinite = sm.draw.best == V::kInf || sm.draw.T == 0.0f;  // the largest, nothing else

  // ---- sums of the cells -----------------------------------------------------------------------
  if (!infinite) order.cell_sums();
  cluster_sync();

  // ---- masses: each CTA of its share of the entries ------------------------------------------
  if (!infinite) {
    const uint32_t ctas = sm.draw.ctas;
    const int share = kEntries / (int)ctas;
    for (int j = tid; j < share; j += kThreads) {
      const int e = (int)rank * share + j;
      uint64_t s[kMostCtas], sum = 0;
      uint32_t n[kMostCtas], number = 0;
#pragma unroll
      for (uint32_t c = 0; c < kMostCtas; ++c) {
        if (c < ctas) {
          s[c] = of_cta(sm.mass + e, c, rank);
          n[c] = of_cta(sm.count + e, c, rank);
        }
      }
#pragma unroll
      for (uint32_t c = 0; c < kMostCtas; ++c) {
        if (c < ctas) {
          sum += s[c];
          number += n[c];
        }
      }
      Weight w = {0, 0};
      if (number) w = order.first(e >= kCells ? e - kCells : kCells - 1 - e, e >= kCells);
      sm.all_mass[j] = number ? mass_of(sum, w) : 0;
      sm.all_first[j] = w.w << 6 | (uint32_t)-w.n;
      sm.all_count[j] = number;
    }
    if (ctas > 1) cluster_sync(); else __syncthreads();
  }

  // ---- filters and draw: the leading CTA -----------------------------------------------------
  if (rank == 0) {
    // two entries a thread, and the sums of all before them
    uint64_t sums[2] = {0, 0};
    uint32_t counts[2] = {0, 0};
    if (!infinite) {
      const uint32_t share = kEntries / sm.draw.ctas, c = 2 * tid / share;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t j = 2 * tid + h - c * share;
        sums[h] = of_cta(sm.all_mass + j, c, 0);
        counts[h] = of_cta(sm.all_count + j, c, 0);
      }
    }
    const uint64_t m0 = sums[0], m1 = sums[1];
    const uint32_t c0 = counts[0], c1 = counts[1];
    uint64_t m = m0 + m1;
    uint32_t c = c0 + c1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t mm = __shfl_up_sync(0xffffffffu, m, o);
      const uint32_t cc = __shfl_up_sync(0xffffffffu, c, o);
      if (lane >= o) {
        m += mm;
        c += cc;
      }
    }
    if (lane == 31) {
      sm.scan_mass[warp] = m;
      sm.scan_count[warp] = c;
    }
    __syncthreads();
    const uint64_t wm = lane < warp ? sm.scan_mass[lane] : 0;
    m += warp_sum(wm);
    c += __reduce_add_sync(0xffffffffu, lane < warp ? sm.scan_count[lane] : 0);
    sm.mass[2 * tid + 1] = m - m1;
    sm.count[2 * tid + 1] = c - c1;
    sm.mass[2 * tid + 2] = m;
    sm.count[2 * tid + 2] = c;
    if (lane == 31) {
      sm.upto_mass[warp] = m;
      sm.upto_count[warp] = c;
    }
    if (tid == 0) {
      sm.mass[0] = 0;
      sm.count[0] = 0;
    }
    __syncthreads();
    if (warp == 0) {
      uint32_t kept, bits, skip;
      float logprob;
      if (infinite) {  // equal weights
        uint32_t n, none;
        bits = sm.draw.best;
        order.counted(bits & 0x7fffu, n, none);
        n = bits & 0x8000u ? none : n;
        kept = sm.draw.T == 0.0f ? 1 : sm.draw.k > 0 ? min((uint32_t)sm.draw.k, n) : n;
        bool more = false;
        if (sm.draw.top_p < 1.0f) kept = max(1u, (uint32_t)part_of(kept, sm.draw.top_p, more) + more);
        skip = (uint32_t)part_of(kept, sm.draw.u, more);
        logprob = 0.0f - logf((float)kept);
      } else {
        uint32_t at = 0xffffffffu;
        kept = sm.count[kEntries];
        uint64_t mass = sm.mass[kEntries];
        const float largest = V::number(sm.draw.best);
        bits = skip = 0;
#pragma unroll 1
        for (int step = 0; step < 4; ++step) {  // top-k, top-p, min-p, the draw
          uint64_t want = 0;
          uint32_t want_n = 0;
          int32_t value = -1;
          if (step == 0) {
            if (sm.draw.k == 0 || (uint32_t)sm.draw.k >= kept) continue;
            want_n = sm.draw.k;
          } else if (step == 2) {
            if (!(sm.draw.min_p > 0.0f)) continue;
            value = (int32_t)least_kept<FP16>(largest, sm.draw.T, sm.draw.min_p);
          } else {
            const float share = step == 1 ? sm.draw.top_p : sm.draw.u;
            if (step == 1 && !(share < 1.0f)) continue;
            bool more;
            want = part_of(mass, share, more);
            want = max((uint64_t)1, want + (more || step == 3));
          }
          const Place x = order.find(want, want_n, value);
          if (step == 3) {
            bits = order.bits_at(x.at);
            skip = x.before;
          } else if (step < 2 || x.at < at) {
            at = x.at;
            kept = x.count;
            mass = x.mass;
          }
        }
        logprob = log_share(V::number(bits), largest, sm.draw.T, mass);
      }
      if (lane == 0) {
        if (p.logprob) p.logprob[i] = logprob;
        if (p.kept) p.kept[i] = (int32_t)kept;
        for (uint32_t c = 0; c < sm.draw.ctas; ++c) {
          const uint32_t w = of_cta(hist + place_of(bits & 0x7fffu), c, 0);
          const uint32_t here = bits == 0 ? (w & 0xffffu) + (w >> 16) : bits & 0x8000u ? w >> 16 : w & 0xffffu;
          if (skip < here) {
            st_cluster(cluster_smem_addr(&sm.found, c), bits);
            st_cluster(cluster_smem_addr(&sm.found_rank, c), skip);
            break;
          }
          skip -= here;
        }
      }
    }
  }
  cluster_sync();

  // ---- where it stands: the CTA whose part has it ----------------------------------------------
  if (sm.found != 0xffffu) find_place<FP16>(p.tokens + i, sm);
}

// The next draw that is left, which is then this cluster's; -1 if there is none.  Clusters walk all
// draws, each from a place of its own; `from` is how far this one is.  By the leading CTA.
__device__ __forceinline__ int32_t claim(const SampleParams& p, Shared& sm, int32_t live,
                                         int64_t begin, int64_t& from) {
  const int tid = threadIdx.x;
  const auto at = [&](int64_t step) {
    const int64_t i = begin + step;
    return (int32_t)(i < live ? i : i - live);
  };
  while (from < live) {
    __syncthreads();
    if (tid == 0) sm.pending = kThreads;
    __syncthreads();
    const bool left = from + tid < live && __ldcg(p.tokens + at(from + tid)) == kPending;
    const unsigned m = __ballot_sync(0xffffffffu, left);
    if ((tid & 31) == 0 && m) atomicMin(&sm.pending, tid + __ffs(m) - 1);
    __syncthreads();
    const int32_t step = sm.pending;
    if (step == kThreads) {
      from += kThreads;
      continue;
    }
    if (tid == 0) {
      const int32_t i = at(from + step);
      sm.next = atomicCAS(p.tokens + i, kPending, kClaimed) == kPending ? i : -1;
    }
    __syncthreads();
    from += step + 1;
    if (sm.next >= 0) return sm.next;
  }
  return -1;
}

// The draws that are left, one after the other.
template <bool FP16>
__global__ void __launch_bounds__(kThreads, 1) order_kernel(const SampleParams p) {
  extern __shared__ uint4 sample_smem[];
  uint32_t* hist = reinterpret_cast<uint32_t*>(sample_smem);
  Shared& sm = *reinterpret_cast<Shared*>(sample_smem + kMags / 4);
  const int tid = threadIdx.x;
  uint32_t ctas;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
  const int32_t cluster = blockIdx.x / ctas, clusters = gridDim.x / ctas;
  if (tid < 129) {
    sm.hi[tid] = kPowers.hi[tid];
    sm.lo[tid] = kPowers.lo[tid];
  }
  pdl_wait();
  pdl_trigger();
  const int32_t live = p.n_dev ? min(__ldg(p.n_dev), p.n) : p.n;
  const int64_t begin = (int64_t)live * cluster / clusters;
  const bool own = p.all || live <= clusters;  // draws of its own: `cluster`, and so on
  int64_t from = own ? cluster : 0;
  for (;;) {  // (one place that draws: its code is large)
    int32_t i = -1;
    if (own) {
      if (from < live && (p.all || __ldcg(p.tokens + from) == kPending)) i = (int32_t)from;
      from += clusters;
    } else {
      if (cluster_ctarank() == 0) {
        i = claim(p, sm, live, begin, from);
        if (tid == 0) sm.next = i;
      }
      cluster_sync();
      i = (int32_t)ld_cluster(cluster_smem_addr(&sm.next, 0));
    }
    if (i < 0) break;
    draw_row<FP16>(p, i, hist, sm, sample_smem);
  }
  cluster_sync();  // nobody leaves while it is read
}

// A launch of clusters of `ctas` CTAs, with programmatic stream serialization.
struct Clusters {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  Clusters(int64_t clusters, int32_t ctas, int threads, size_t smem, cudaStream_t stream) {
    cfg.gridDim = dim3((unsigned)(clusters * ctas));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
  }
};

constexpr size_t kOrderSmem = kMags * 4 + sizeof(Shared);

// How many clusters of 1, 2, 4 and 8 CTAs of order_kernel a device holds.
std::atomic<int32_t> g_most[kMaxDeviceOrdinals][4];

hs_status order_setup(int dev) {
  for (const auto f : {order_kernel<false>, order_kernel<true>}) {
    const hs_status st = cuda_fail(
        cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kOrderSmem),
        "sample shared memory");
    if (st != HS_OK) return st;
  }
  for (int i = 0; i < 4; ++i) {
    int most = 0;
    const Clusters c(1, 1 << i, kThreads, kOrderSmem, nullptr);
    const hs_status st = cuda_fail(
        cudaOccupancyMaxActiveClusters(&most, order_kernel<false>, &c.cfg), "sample clusters");
    if (st != HS_OK) return st;
    g_most[dev][i].store(most > 1 ? most : 1, std::memory_order_relaxed);
  }
  return HS_OK;
}

}  // namespace

hs_status launch_sample(SampleParams p, bool fp16, cudaStream_t stream) {
  p.err = device_error_word();
  if (!p.err) return fail(HS_ERR_CUDA, "could not resolve the device error word");
  const int dev = device_ordinal() < 0 ? 0 : device_ordinal();
  static std::atomic<uint64_t> configured{0};
  const hs_status st = once_per_device(configured, [dev] { return order_setup(dev); });
  if (st != HS_OK) return st;
  const int32_t vecs = (p.vocab + 7 + 7) / 8;
  const auto most = [dev](int log2) {
    return (int64_t)g_most[dev][log2].load(std::memory_order_relaxed);
  };
  // A row that is all head leaves nothing.
  p.whole = p.vocab <= kHeadMost;
  p.either = vecs > 1024;
  // order_kernel: as few CTAs a row as its counts allow.
  int log2 = 0;
  while ((vecs + (1 << log2) - 1) >> log2 > kMostVecs) ++log2;
  // By itself where it takes the draws in two rounds at most: a round is 16 us (from 4000 logits)
  // to 25 (from 128,000), and head_kernel's 8 to 15 come on top for any draw that is left.  Few
  // draws leave none, most of the time, and neither do small vocabularies.  After the heads and
  // alone, us, draws with settings of their own (and all with top-p 0.95 and no top-k, which leave
  // many): 64 draws from 4000 logits 13 and 18 (13 and 17), 8000 16 and 19 (16 and 17), 16,000 24
  // and 19 (29 and 17), 32,000 38 and 20 (41 and 18), 128,000 44 and 26 (106 and 25); 600 draws,
  // four rounds, from 32,000 52 and 79 (67 and 74).
  // A number of draws cannot tell these two kinds apart, so the rule is wrong for one of them at
  // its ends: 2 draws from 128,000 13 and 21 (34 and 20: the heads are taken), 4 of them 15 and 22
  // (34 and 20: the order); 304, which are four rounds there, 72 and 94 (143 and 91: the heads), 600
  // 104 and 183 (266 and 178: the heads).
  p.all = p.n >= 4 && p.either && p.n <= 2 * most(log2);
  if (!p.all) {
    // The heads: several CTAs share an SM; more of them a row where rows are few.
    int32_t heads = 1;
    while (heads < kMostCtas && (int64_t)p.n * heads * 2 <= 4 * num_sms() &&
           vecs / heads > 2 * kHeadThreads)
      heads *= 2;
    const Clusters c(p.n, heads, kHeadThreads, 0, stream);
    cudaLaunchKernelEx(&c.cfg, fp16 ? head_kernel<true> : head_kernel<false>, p);
    count_launches(1);
    if (p.whole) return cuda_fail(cudaGetLastError(), "sample launch");
  }
  // More CTAs a row where the draws do not fill them: about a sixth of all is left at most.
  const int64_t rows = p.all ? p.n : p.n / 6;
  while (1 << log2 < kMostCtas && rows <= most(log2 + 1) && vecs >> log2 > 1024) ++log2;
  const Clusters c(p.n < most(log2) ? p.n : most(log2), 1 << log2, kThreads, kOrderSmem, stream);
  cudaLaunchKernelEx(&c.cfg, fp16 ? order_kernel<true> : order_kernel<false>, p);
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "sample launch");
}

}  // namespace hs
