// Block tables and slot maps of the paged cache (hs_kv_tables), and the way back of a finished
// request's blocks (hs_kv_release).
//
// With bt tokens a block, request r's new blocks are numbers first_r = ceil(have_r / bt) up to
// ceil((have_r + fresh_r) / bt) - 1 of its row.  Two exclusive prefix sums over the requests, of
// new tokens (S) and of new blocks (B), place everything else:
//   entry first_r + j of row r is the ring's block number taken + B_r + j;
//   the batch's token t belongs to the last r with S_r <= t, is token p = have_r + t - S_r of its
//   request, and its slot is block(p / bt) * bt + p % bt.
// The inputs are a few numbers a request, so no CTA waits for another: each computes both sums
// over all requests into its own shared memory (8 bytes a request) and writes its share of the
// tokens and of the new entries, found by binary search.  One launch; what bounds a decoding
// step's call is the latency of its two dependent reads (64 requests 3.8 us; 1434 prompts with
// 413,000 tokens 9.1, for 1.8 MB).
#include "hs_internal.cuh"

namespace hs {
namespace {

constexpr int kTabThreads = 512;
constexpr int kTabWarps = kTabThreads / 32;
constexpr int kTabPerCta = 2 * kTabThreads;  // tokens and entries for one CTA, at least

struct TabParams {
  const int32_t* have;
  const int32_t* fresh;
  int64_t n_req;
  const int32_t* n_req_dev;
  int32_t bt_log2;
  int32_t* table;
  int32_t width;
  const int32_t* pool;
  int32_t n_blocks;
  const int64_t* cursor;
  int64_t* cursor_out;
  int32_t* starts_out;
  int32_t* lens_out;
  int32_t* slots_out;
  int64_t max_tokens;
  unsigned* err;
};

__device__ __forceinline__ int32_t live_requests(int64_t n_req, const int32_t* n_req_dev) {
  if (!n_req_dev) return (int32_t)n_req;
  const int32_t c = __ldg(n_req_dev);
  return (int32_t)(c < 0 ? 0 : (c > n_req ? n_req : c));
}

// Exclusive prefix of (a, b) over the block's threads; totals in ta, tb.
__device__ __forceinline__ void block_scan2(int64_t& a, int64_t& b, int64_t& ta, int64_t& tb) {
  __shared__ int64_t sa[kTabWarps], sb[kTabWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t x = a, y = b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) {
      x += u;
      y += v;
    }
  }
  if (lane == 31) {
    sa[warp] = x;
    sb[warp] = y;
  }
  __syncthreads();
  ta = tb = 0;
  int64_t ba = 0, bb = 0;
#pragma unroll
  for (int w = 0; w < kTabWarps; ++w) {
    if (w == warp) {
      ba = ta;
      bb = tb;
    }
    ta += sa[w];
    tb += sb[w];
  }
  a = ba + x - a;
  b = bb + y - b;
}

__device__ __forceinline__ int32_t clip31(int64_t x) {
  return (int32_t)(x < 0x7fffffffLL ? x : 0x7fffffffLL);
}

// The last r in [0, n) with pre[r] <= x, where pre[0] = 0 <= x < pre[n].
__device__ __forceinline__ int32_t find_request(const int32_t* pre, int32_t n, int32_t x) {
  int32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (pre[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// A request's counts; one that its row of the table cannot hold has none.
__device__ __forceinline__ bool request(const TabParams& p, int32_t r, int32_t& have,
                                        int32_t& fresh) {
  have = __ldg(p.have + r);
  fresh = __ldg(p.fresh + r);
  if (have < 0 || fresh < 0 || (int64_t)have + fresh > ((int64_t)p.width << p.bt_log2)) {
    have = fresh = 0;
    return false;
  }
  return true;
}

__device__ __forceinline__ int32_t blocks_of(int64_t tokens, int log2) {
  return (int32_t)((tokens + (1 << log2) - 1) >> log2);
}

__global__ void __launch_bounds__(kTabThreads) kv_tables_kernel(const TabParams p) {
  extern __shared__ int32_t pre[];  // tokens before each request, then new blocks before it
  pdl_wait();
  pdl_trigger();
  const int32_t R = live_requests(p.n_req, p.n_req_dev);
  const int64_t taken = __ldg(p.cursor), given = __ldg(p.cursor + 1);
  int32_t* pre_t = pre;
  int32_t* pre_b = pre + R + 1;
  const int tid = threadIdx.x;
  const int32_t per = (R + kTabThreads - 1) / kTabThreads;
  const int32_t r0 = min(tid * per, R), r1 = min(r0 + per, R);
  int64_t t = 0, b = 0, total_t, total_b;
  unsigned bad = 0;
  for (int32_t r = r0; r < r1; ++r) {
    int32_t have, fresh;
    if (!request(p, r, have, fresh)) bad = kErrInvalidArg;
    t += fresh;
    b += blocks_of((int64_t)have + fresh, p.bt_log2) - blocks_of(have, p.bt_log2);
  }
  block_scan2(t, b, total_t, total_b);
  for (int32_t r = r0; r < r1; ++r) {
    int32_t have, fresh;
    request(p, r, have, fresh);
    pre_t[r] = clip31(t);
    pre_b[r] = clip31(b);
    t += fresh;
    b += blocks_of((int64_t)have + fresh, p.bt_log2) - blocks_of(have, p.bt_log2);
  }
  if (tid == 0) {
    pre_t[R] = clip31(total_t);
    pre_b[R] = clip31(total_b);
  }
  __syncthreads();

  // The ring: what is left of it, and where it begins.
  int64_t left = given - taken;
  if (taken < 0 || left < 0 || left > p.n_blocks) {
    left = 0;
    bad = kErrInvalidArg;
  }
  const int32_t avail = (int32_t)(total_b < left ? total_b : left);
  if (avail < total_b || total_t > p.max_tokens) bad = kErrInvalidArg;
  const int32_t ring = taken < 0 ? 0 : (int32_t)(taken % p.n_blocks);
  const auto ring_block = [&](int32_t j) -> int32_t {  // j < avail; -1 if the entry is no block
    int64_t at = (int64_t)ring + j;
    if (at >= p.n_blocks) at -= p.n_blocks;
    const int32_t id = __ldg(p.pool + at);
    return (uint32_t)id < (uint32_t)p.n_blocks ? id : -1;
  };

  const int64_t me = (int64_t)blockIdx.x * kTabThreads + tid;
  const int64_t all = (int64_t)gridDim.x * kTabThreads;
  const int32_t n_tok = (int32_t)(total_t < p.max_tokens ? total_t : p.max_tokens);
  for (int64_t i = me; i < p.max_tokens; i += all) {
    int32_t slot = -1;
    if (i < n_tok) {
      const int32_t r = find_request(pre_t, R, (int32_t)i);
      const int32_t have = __ldg(p.have + r);
      const int64_t pos = (int64_t)have + ((int32_t)i - pre_t[r]);
      const int32_t blk = (int32_t)(pos >> p.bt_log2), first = blocks_of(have, p.bt_log2);
      int32_t id = -1;
      if (blk < first) {
        id = p.table[(int64_t)r * p.width + blk];
        if ((uint32_t)id >= (uint32_t)p.n_blocks) {
          id = -1;
          bad = kErrInvalidArg;
        }
      } else {
        const int64_t j = (int64_t)pre_b[r] + (blk - first);
        if (j < avail) id = ring_block((int32_t)j);
      }
      if (id >= 0) slot = (id << p.bt_log2) + (int32_t)(pos & ((1 << p.bt_log2) - 1));
    }
    p.slots_out[i] = slot;
  }
  const int32_t n_new = clip31(total_b);
  for (int64_t i = me; i < n_new; i += all) {
    const int32_t r = find_request(pre_b, R, (int32_t)i);
    const int32_t have = __ldg(p.have + r);
    int32_t id = -1;
    if (i < avail) {
      id = ring_block((int32_t)i);
      if (id < 0) bad = kErrInvalidArg;
    }
    p.table[(int64_t)r * p.width + blocks_of(have, p.bt_log2) + ((int32_t)i - pre_b[r])] = id;
  }
  for (int64_t r = me; r <= p.n_req; r += all) {
    p.starts_out[r] = pre_t[r < R ? r : R];
    if (r < p.n_req) {
      int32_t have = 0, fresh = 0, len = 0;
      if (r < R) {
        request(p, (int32_t)r, have, fresh);
        const int64_t want = (int64_t)have + fresh;
        const int32_t short_of = max(pre_b[r + 1] - max(avail, pre_b[r]), 0);
        const int64_t most = (int64_t)(blocks_of(want, p.bt_log2) - short_of) << p.bt_log2;
        len = (int32_t)(want < most ? want : most);
      }
      p.lens_out[r] = len;
    }
  }
  if (me == 0) {
    p.cursor_out[0] = taken + avail;
    p.cursor_out[1] = given;
  }
  if (bad) set_error(p.err, bad);
}

struct ReleaseParams {
  const int32_t* lens;
  int64_t n_req;
  const int32_t* n_req_dev;
  int32_t bt_log2;
  const int32_t* table;
  int32_t width;
  int32_t* pool;
  int32_t n_blocks;
  const int64_t* cursor;
  int64_t* cursor_out;
  unsigned* err;
};

// One CTA.  Requests are counted over valid entries only, so an entry that is no block leaves no
// hole in the ring: a thread walks its requests' entries twice, to count and to write.
__global__ void __launch_bounds__(kTabThreads) kv_release_kernel(const ReleaseParams p) {
  pdl_wait();
  pdl_trigger();
  const int32_t R = live_requests(p.n_req, p.n_req_dev);
  const int64_t taken = __ldg(p.cursor), given = __ldg(p.cursor + 1);
  const int tid = threadIdx.x, lane = tid & 31;
  unsigned bad = 0;
  // A warp per request and round, kTabWarps requests at a time, in the requests' order.
  __shared__ int32_t counts[kTabWarps];
  int64_t done = 0;
  int64_t room = (int64_t)p.n_blocks - (given - taken);
  if (taken < 0 || given < taken || room < 0) {
    room = 0;
    bad = kErrInvalidArg;
  }
  for (int32_t base = 0; base < R; base += kTabWarps) {
    const int32_t r = base + (tid >> 5);
    int32_t n = 0;
    if (r < R) {
      const int32_t len = __ldg(p.lens + r);
      if (len < 0 || len > ((int64_t)p.width << p.bt_log2)) bad = kErrInvalidArg;
      else n = blocks_of(len, p.bt_log2);
    }
    const int32_t* row = p.table + (int64_t)r * p.width;
    int32_t valid = 0;
    for (int32_t j0 = 0; j0 < n; j0 += 32) {
      const bool in = j0 + lane < n;
      const bool ok = in && (uint32_t)__ldg(row + j0 + lane) < (uint32_t)p.n_blocks;
      if (in && !ok) bad = kErrInvalidArg;
      valid += __popc(__ballot_sync(0xffffffffu, ok));
    }
    if (lane == 0) counts[tid >> 5] = valid;
    __syncthreads();
    int64_t at = done;
    for (int w = 0; w < kTabWarps; ++w) {
      if (w < (tid >> 5)) at += counts[w];
      done += counts[w];
    }
    for (int32_t j0 = 0; j0 < n; j0 += 32) {
      const int32_t id = j0 + lane < n ? __ldg(row + j0 + lane) : -1;
      const bool ok = (uint32_t)id < (uint32_t)p.n_blocks;
      const unsigned m = __ballot_sync(0xffffffffu, ok);
      const int64_t mine = at + __popc(m & lanemask_lt());
      if (ok && mine < room) p.pool[(given + mine) % p.n_blocks] = id;
      at += __popc(m);
    }
    __syncthreads();
  }
  if (done > room) {
    done = room;
    bad = kErrInvalidArg;
  }
  if (tid == 0) {
    p.cursor_out[0] = taken;
    p.cursor_out[1] = given + done;
  }
  if (bad) set_error(p.err, bad);
}

}  // namespace

hs_status launch_kv_tables(const int32_t* have, const int32_t* fresh, int64_t n_req,
                           const int32_t* n_req_dev, int32_t bt_log2, int32_t* table,
                           int32_t width, const int32_t* pool, int64_t n_blocks,
                           const int64_t* cursor, int64_t* cursor_out, int32_t* starts_out,
                           int32_t* lens_out, int32_t* slots_out, int64_t max_tokens,
                           cudaStream_t stream) {
  unsigned* err = device_error_word();
  if (!err) return fail(HS_ERR_CUDA, "could not resolve the device error word");
  const TabParams p{have, fresh, n_req, n_req_dev, bt_log2, table, width, pool, (int32_t)n_blocks,
                    cursor, cursor_out, starts_out, lens_out, slots_out, max_tokens, err};
  const size_t smem = (size_t)(n_req + 1) * 8;
  if (smem > 48 * 1024) {
    static std::atomic<uint64_t> configured{0};
    const hs_status st = once_per_device(configured, [] {
      return cuda_fail(cudaFuncSetAttribute(kv_tables_kernel,
                                            cudaFuncAttributeMaxDynamicSharedMemorySize,
                                            (HS_KV_MAX_REQUESTS + 1) * 8),
                       "kv_tables shared memory");
    });
    if (st != HS_OK) return st;
  }
  int64_t grid = ((max_tokens > n_req ? max_tokens : n_req) + kTabPerCta - 1) / kTabPerCta;
  if (grid < 1) grid = 1;
  if (grid > num_sms()) grid = num_sms();
  launch_pdl(kv_tables_kernel, dim3((unsigned)grid), dim3(kTabThreads), smem, stream, p);
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "kv_tables launch");
}

hs_status launch_kv_release(const int32_t* lens, int64_t n_req, const int32_t* n_req_dev,
                            int32_t bt_log2, const int32_t* table, int32_t width, int32_t* pool,
                            int64_t n_blocks, const int64_t* cursor, int64_t* cursor_out,
                            cudaStream_t stream) {
  unsigned* err = device_error_word();
  if (!err) return fail(HS_ERR_CUDA, "could not resolve the device error word");
  const ReleaseParams p{lens, n_req, n_req_dev, bt_log2, table, width, pool, (int32_t)n_blocks,
                        cursor, cursor_out, err};
  launch_pdl(kv_release_kernel, dim3(1), dim3(kTabThreads), 0, stream, p);
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "kv_release launch");
}

}  // namespace hs
