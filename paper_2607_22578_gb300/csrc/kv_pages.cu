// Blocks of the paged cache that several requests hold: requests that go on as several
// (hs_kv_fork), the copy of listed blocks (hs_kv_copy), the way back of blocks that nobody holds
// any more (hs_kv_release_shared) and the move of all blocks in use to the low end of the cache
// (hs_kv_compact).
//
// shared[b] counts the requests that hold block b beyond the first, so a block that hs_kv_tables
// gave out has 0 and needs no entry there.  Only full blocks are shared: a request's last, partly
// filled block is its own, and hs_kv_append never writes to another's.
#include "hs_internal.cuh"

namespace hs {
namespace {

constexpr int kForkThreads = 512;
constexpr int kPageThreads = 1024;
constexpr int kPageWarps = kPageThreads / 32;
constexpr int kPageCtas = 8;  // one cluster: its barrier orders a pass before the next

__device__ __forceinline__ int32_t live_requests(int64_t n_req, const int32_t* n_req_dev) {
  if (!n_req_dev) return (int32_t)n_req;
  const int32_t c = __ldg(n_req_dev);
  return (int32_t)(c < 0 ? 0 : (c > n_req ? n_req : c));
}

__device__ __forceinline__ int32_t blocks_of(int64_t tokens, int log2) {
  return (int32_t)((tokens + (1 << log2) - 1) >> log2);
}

// ---- fork ----------------------------------------------------------------------------------
// Pair i of valid ones gives row d = dst[i] the first F = floor(L / bt) blocks of row s = src[i],
// L = lens[s], and where L is no multiple of bt the ring's block number taken + B_i, B_i the
// pairs before i that need one.  As in hs_kv_tables no CTA waits for another: each finds out
// which pairs are valid and the prefix sum of those that need a block in its own shared memory
// (8 bytes a row and pair), and does its share of the rows.  Counts go up by atomic additions,
// whose order changes nothing.  A chain of four round trips bounds it (pair, lengths, table, the
// ring), so a thread looks four pairs up together: 2048 pairs 7.0 -> 5.2 us, 64 pairs 4.6.

struct ForkParams {
  const int32_t* src;
  const int32_t* dst;
  int32_t n;
  const int32_t* lens;
  int32_t* lens_out;
  int32_t n_req;
  int32_t bt_log2;
  int32_t* table;
  int32_t width;
  int32_t* shared;
  const int32_t* pool;
  int32_t n_blocks;
  const int64_t* cursor;
  int64_t* cursor_out;
  int32_t* source;
  int32_t* target;
  int32_t* tokens;
  const int32_t* n_req_dev;
  int32_t* n_req_out;  // or NULL
  unsigned* err;
};

// Exclusive prefix of x over the block's threads.
__device__ __forceinline__ int32_t fork_scan(int32_t x, int32_t& total) {
  __shared__ int32_t sums[kForkThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t y = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t u = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) y += u;
  }
  if (lane == 31) sums[warp] = y;
  __syncthreads();
  int32_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kForkThreads / 32; ++w) {
    if (w == warp) before = total;
    total += sums[w];
  }
  return before + y - x;
}

// Whether pair i makes a row, of how many tokens, and which block's rest it needs (-1: none).
__device__ __forceinline__ bool fork_pair(const ForkParams& p, const int32_t* first, int32_t i,
                                          int32_t& s, int32_t& d, int32_t& len, int32_t& tail,
                                          unsigned& bad) {
  s = __ldg(p.src + i);
  d = __ldg(p.dst + i);
  tail = -1;
  if (d == -1 || s == d) return false;
  if ((uint32_t)s >= (uint32_t)p.n_req || (uint32_t)d >= (uint32_t)p.n_req || first[d] != i ||
      __ldg(p.lens + d) != 0) {
    bad = kErrInvalidArg;
    return false;
  }
  len = __ldg(p.lens + s);
  if (len < 0 || len > ((int64_t)p.width << p.bt_log2)) {
    bad = kErrInvalidArg;
    return false;
  }
  if (len & ((1 << p.bt_log2) - 1)) {
    // (row s is not written by this call: it has tokens)
    tail = __ldg(p.table + (int64_t)s * p.width + (len >> p.bt_log2));
    if ((uint32_t)tail >= (uint32_t)p.n_blocks) {
      tail = -1;
      bad = kErrInvalidArg;
    }
  }
  return true;
}

__global__ void __launch_bounds__(kForkThreads) kv_fork_kernel(const ForkParams p) {
  extern __shared__ int32_t fork_smem[];
  __shared__ int32_t rows;                // up to the last that is made
  int32_t* first = fork_smem;             // the first pair that names a row as its own
  int32_t* before = fork_smem + p.n_req;  // new blocks before each pair
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31;
  const int64_t taken = __ldg(p.cursor), given = __ldg(p.cursor + 1);
  unsigned bad = 0;
  int32_t last = 0;
  if (tid == 0) rows = 0;
  for (int32_t r = tid; r < p.n_req; r += kForkThreads) first[r] = 0x7fffffff;
  __syncthreads();
  for (int32_t i = tid; i < p.n; i += kForkThreads) {
    const int32_t s = __ldg(p.src + i), d = __ldg(p.dst + i);
    if (s != d && (uint32_t)d < (uint32_t)p.n_req) atomicMin(first + d, i);
  }
  __syncthreads();
  // Which pairs need a block: four a thread at a time, so that their loads are on the way together.
  for (int32_t i0 = tid; i0 < p.n; i0 += 4 * kForkThreads) {
    int32_t s[4], d[4], own[4], len[4], tail[4];
    bool makes[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int32_t i = i0 + h * kForkThreads;
      makes[h] = i < p.n;
      s[h] = makes[h] ? __ldg(p.src + i) : 0;
      d[h] = makes[h] ? __ldg(p.dst + i) : -1;
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      makes[h] = d[h] != -1 && s[h] != d[h];
      if (makes[h] && ((uint32_t)s[h] >= (uint32_t)p.n_req || (uint32_t)d[h] >= (uint32_t)p.n_req ||
                       first[d[h]] != i0 + h * kForkThreads)) {
        makes[h] = false;
        bad = kErrInvalidArg;
      }
      own[h] = makes[h] ? __ldg(p.lens + d[h]) : 0;
      len[h] = makes[h] ? __ldg(p.lens + s[h]) : 0;
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      if (own[h] != 0 || len[h] < 0 || len[h] > ((int64_t)p.width << p.bt_log2)) {
        bad = kErrInvalidArg;
        len[h] = 0;
      } else if (makes[h]) {
        last = max(last, d[h] + 1);
      }
      tail[h] = -1;
      if (len[h] & ((1 << p.bt_log2) - 1))
        tail[h] = __ldg(p.table + (int64_t)s[h] * p.width + (len[h] >> p.bt_log2));
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int32_t i = i0 + h * kForkThreads;
      const bool needs = (uint32_t)tail[h] < (uint32_t)p.n_blocks;
      if (!needs && (len[h] & ((1 << p.bt_log2) - 1))) bad = kErrInvalidArg;
      if (i < p.n) before[i] = needs;
    }
  }
  if (p.n_req_out) {
    last = __reduce_max_sync(0xffffffffu, last);
    if (lane == 0) atomicMax(&rows, last);
  }
  __syncthreads();
  const int32_t per = (p.n + kForkThreads - 1) / kForkThreads;
  const int32_t i0 = min(tid * per, p.n), i1 = min(i0 + per, p.n);
  int32_t need = 0, total, s, d, len, tail;
  for (int32_t i = i0; i < i1; ++i) need += before[i];
  int32_t at = fork_scan(need, total);
  for (int32_t i = i0; i < i1; ++i) {
    const int32_t needs = before[i];
    before[i] = at;
    at += needs;
  }
  __syncthreads();

  int64_t left = given - taken;
  if (taken < 0 || left < 0 || left > p.n_blocks) {
    left = 0;
    bad = kErrInvalidArg;
  }
  const int32_t avail = (int32_t)(total < left ? total : left);
  if (avail < total) bad = kErrInvalidArg;
  const int32_t ring = taken < 0 ? 0 : (int32_t)(taken % p.n_blocks);
  const auto new_block = [&](int32_t j) -> int32_t {  // -1 past what is left, or if it is none
    if (j >= avail) return -1;
    int64_t k = (int64_t)ring + j;
    if (k >= p.n_blocks) k -= p.n_blocks;
    const int32_t id = __ldg(p.pool + k);
    return (uint32_t)id < (uint32_t)p.n_blocks ? id : -1;
  };
  const int32_t me = blockIdx.x * kForkThreads + tid, all = gridDim.x * kForkThreads;
  for (int32_t r = me; r < p.n_req; r += all) {
    const int32_t i = first[r];
    int32_t out = __ldg(p.lens + r);
    unsigned seen = 0;
    if (i != 0x7fffffff && fork_pair(p, first, i, s, d, len, tail, seen))
      out = tail >= 0 && new_block(before[i]) < 0 ? len & ~((1 << p.bt_log2) - 1) : len;
    p.lens_out[r] = out;
  }
  // A warp for each pair.
  for (int32_t i = me >> 5; i < p.n; i += all >> 5) {
    unsigned seen = 0;
    const bool makes = fork_pair(p, first, i, s, d, len, tail, seen);
    int32_t fresh = -1;
    if (makes && tail >= 0) {
      fresh = new_block(before[i]);
      if (fresh < 0) bad = kErrInvalidArg;
    }
    if (lane == 0) {
      const bool copies = fresh >= 0;
      p.source[i] = copies ? tail : -1;
      p.target[i] = copies ? fresh : -1;
      p.tokens[i] = copies ? len & ((1 << p.bt_log2) - 1) : 0;
    }
    if (!makes) continue;
    const int32_t full = len >> p.bt_log2;
    const int32_t* from = p.table + (int64_t)s * p.width;
    int32_t* to = p.table + (int64_t)d * p.width;
    for (int32_t j = lane; j < full; j += 32) {
      int32_t id = from[j];
      if ((uint32_t)id < (uint32_t)p.n_blocks) {
        atomicAdd(p.shared + id, 1);
      } else {
        id = -1;
        bad = kErrInvalidArg;
      }
      to[j] = id;
    }
    if (lane == 0 && (len & ((1 << p.bt_log2) - 1))) to[full] = fresh;
  }
  if (me == 0) {
    p.cursor_out[0] = taken + avail;
    p.cursor_out[1] = given;
    if (p.n_req_out) *p.n_req_out = max(live_requests(p.n_req, p.n_req_dev), rows);
  }
  if (bad) set_error(p.err, bad);
}

// ---- copy ----------------------------------------------------------------------------------
// A head's codes of a block are one run of bt * dim bytes.  A warp copies up to 4 KB of one:
// 16 bytes a lane and load, all loads of a piece before its stores.  Memory bounds it: 2030 blocks
// of 128 KB move in 80 us (6.7 TB/s read and written).  32 CTAs an SM in the grid, four of them at a
// time: with 8, which take several pieces in turn, that is 84, and with 128 as well.

constexpr int kCopyThreads = 256;
constexpr int kCopyPiece = 4096;

struct CopyParams {
  uint8_t* codes[2];
  float* scale[2];
  int64_t n_blocks;
  int32_t H;
  int32_t bt;
  int32_t dim;
  int32_t pieces;  // of one run
  const int32_t* source;
  const int32_t* target;
  const int32_t* tokens;
  int64_t n;
  const int32_t* n_dev;
  unsigned* err;
};

__global__ void __launch_bounds__(kCopyThreads) kv_copy_kernel(const CopyParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  int64_t n = p.n;
  if (p.n_dev) {
    const int32_t c = __ldg(p.n_dev);
    n = c < 0 ? 0 : c < n ? c : n;
  }
  const int32_t per = 2 * p.H * p.pieces, run = p.bt * p.dim;
  const int64_t items = n * per;
  unsigned bad = 0;
  for (int64_t it = ((int64_t)blockIdx.x * kCopyThreads + threadIdx.x) >> 5; it < items;
       it += ((int64_t)gridDim.x * kCopyThreads) >> 5) {
    const int64_t i = it / per;
    int32_t rest = (int32_t)(it - i * per);
    const int32_t piece = rest % p.pieces;
    rest /= p.pieces;
    const int32_t h = rest >> 1, x = rest & 1;
    const int32_t s = __ldg(p.source + i), t = __ldg(p.target + i);
    const int32_t tok = p.tokens ? __ldg(p.tokens + i) : p.bt;
    if (s == -1 || t == -1 || s == t) continue;
    if ((uint32_t)s >= (uint64_t)p.n_blocks || (uint32_t)t >= (uint64_t)p.n_blocks || tok < 0 ||
        tok > p.bt) {
      bad = kErrInvalidArg;
      continue;
    }
    if (tok == 0) continue;
    const int64_t from = (int64_t)s * p.H + h, to = (int64_t)t * p.H + h;
    if (piece == 0 && lane == 0) p.scale[x][to] = p.scale[x][from];
    const int32_t bytes = min(tok * p.dim - piece * kCopyPiece, kCopyPiece);
    const uint8_t* a = p.codes[x] + from * run + piece * kCopyPiece;
    uint8_t* b = p.codes[x] + to * run + piece * kCopyPiece;
    uint4 v[kCopyPiece / 512];
#pragma unroll
    for (int j = 0; j < kCopyPiece / 512; ++j)
      if (j * 512 + lane * 16 < bytes)
        v[j] = *reinterpret_cast<const uint4*>(a + j * 512 + lane * 16);
#pragma unroll
    for (int j = 0; j < kCopyPiece / 512; ++j)
      if (j * 512 + lane * 16 < bytes) *reinterpret_cast<uint4*>(b + j * 512 + lane * 16) = v[j];
  }
  if (bad) set_error(p.err, bad);
}

// ---- release and compact -------------------------------------------------------------------
// Both pass over the table's entries, then over the blocks in order.  Where the CTAs of one
// cluster share that, the cluster's barrier stands between two passes, and also makes what they
// wrote to global memory visible (read again from the second-level cache).

// The sum over the cluster's CTAs before this one and over all, of one number each.
template <int CTAS = kPageCtas>
__device__ __forceinline__ void cluster_sums(int32_t mine, int32_t* slot, int32_t& before,
                                             int32_t& total, int32_t ctas = CTAS) {
  if (threadIdx.x == 0) *slot = mine;
  cluster_sync();
  before = total = 0;
  const uint32_t me = cluster_ctarank();
#pragma unroll
  for (uint32_t c = 0; c < CTAS; ++c) {
    const int32_t x = (int32_t)c < ctas ? (int32_t)ld_cluster(cluster_smem_addr(slot, c)) : 0;
    if (c < me) before += x;
    total += x;
  }
}

// The sum over the block's warps before this one and over all, of one number a warp.
__device__ __forceinline__ void block_sums(int32_t mine, int32_t* slots, int32_t& before,
                                           int32_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
  if (lane == 0) slots[warp] = mine;
  __syncthreads();
  int32_t x = slots[lane];
  const int32_t own = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t u = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += u;
  }
  before = __shfl_sync(0xffffffffu, x - own, warp);
  total = __shfl_sync(0xffffffffu, x, 31);
}

// Calls f(id) for the entries of lens[r] tokens of each request, one warp a request.
template <class F>
__device__ __forceinline__ void each_entry(const int32_t* lens, int32_t R, int bt_log2,
                                           const int32_t* table, int32_t width, int32_t n_blocks,
                                           unsigned& bad, F&& f) {
  const int lane = threadIdx.x & 31;
  const int32_t warp = (int32_t)cluster_ctarank() * kPageWarps + (threadIdx.x >> 5);
  for (int32_t r = warp; r < R; r += kPageCtas * kPageWarps) {
    const int32_t len = __ldg(lens + r);
    if (len < 0 || len > ((int64_t)width << bt_log2)) {
      bad = kErrInvalidArg;
      continue;
    }
    const int32_t n = blocks_of(len, bt_log2);
    for (int32_t j = lane; j < n; j += 32) {
      const int64_t at = (int64_t)r * width + j;
      const int32_t id = table[at];
      if ((uint32_t)id < (uint32_t)n_blocks) f(at, id);
      else bad = kErrInvalidArg;
    }
  }
}

// This warp's range of the blocks: contiguous, in the order of CTAs and warps.
__device__ __forceinline__ void warp_range(int32_t n, int32_t& a, int32_t& b) {
  const int32_t warps = kPageCtas * kPageWarps;
  const int32_t w = (int32_t)cluster_ctarank() * kPageWarps + (threadIdx.x >> 5);
  const int64_t per = (((int64_t)n + warps - 1) / warps + 31) / 32 * 32;
  a = (int32_t)min((int64_t)n, w * per);
  b = (int32_t)min((int64_t)n, (w + 1) * per);
}

struct ShareParams {
  const int32_t* lens;
  int64_t n_req;
  const int32_t* n_req_dev;
  int32_t bt_log2;
  const int32_t* table;
  int32_t width;
  const int32_t* shared;
  int32_t* shared_out;
  int32_t* pool;
  int32_t n_blocks;
  const int64_t* cursor;
  int64_t* cursor_out;
  unsigned* err;
};

// Each entry takes one from its block's count; a block whose count falls below 0 has no holder
// left and goes into the ring, in the order of the blocks' numbers: the same whatever the order of
// the additions.  Where both are few one CTA holds the counts in shared memory.  Otherwise the
// copy of the counts and the additions are kernels of all SMs (scattered additions are one a clock
// and SM), and the blocks in order are one cluster's work, 32 a thread at a time, held in registers
// between the count and the ring.  Latency bounds all of it: 16 of 64 requests in 8192 blocks 6.8
// us (8.4 as one cluster), 108,000 entries in 262,144 blocks 14.6 us in three kernels (41 as one
// cluster of eight), 290,000 in 518,048 blocks 20 (29 with a cluster of eight).  Those 16 requests in
// caches of 16,384, 32,768, 65,536, 262,144 and 524,288 blocks: 11.9, 29.4, 9.7, 10.4 and 11.1 us.  The
// first two are one CTA's, whose lanes read counts of n_blocks / 1024 blocks each, so that 16 and 32 of
// a warp's meet in one bank.
constexpr int32_t kShareFew = 32768;           // blocks: 128 KB
constexpr int64_t kShareFewEntries = 16384;
constexpr int kShareSteps = 8;  // of 4 blocks a lane, at most
constexpr int kShareCtas = 16;  // of the cluster, or kPageCtas where the device has no such clusters

__global__ void __launch_bounds__(kPageThreads) kv_share_copy_kernel(const ShareParams p) {
  pdl_wait();
  pdl_trigger();
  const int32_t all = gridDim.x * kPageThreads;
  for (int32_t i = blockIdx.x * kPageThreads + threadIdx.x; i < p.n_blocks; i += all)
    p.shared_out[i] = __ldg(p.shared + i);
}

// Takes one from the counts that the entries name, 128 entries of a request a warp at a time.
__device__ __forceinline__ void release_entries(const ShareParams& p, int32_t* counts, int32_t first,
                                                int32_t warps, unsigned& bad) {
  const int32_t R = live_requests(p.n_req, p.n_req_dev);
  const int lane = threadIdx.x & 31;
  const int32_t chunks = (p.width + 127) / 128;
  const int64_t items = (int64_t)R * chunks;
  for (int64_t it = first; it < items; it += warps) {
    const int32_t r = (int32_t)(it / chunks), j0 = (int32_t)(it - (int64_t)r * chunks) * 128;
    const int32_t len = __ldg(p.lens + r);
    if (len < 0 || len > ((int64_t)p.width << p.bt_log2)) {
      bad = kErrInvalidArg;
      continue;
    }
    const int32_t n = blocks_of(len, p.bt_log2);
    const int32_t* row = p.table + (int64_t)r * p.width;
    int32_t id[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int32_t j = j0 + 32 * h + lane;
      id[h] = j < n ? __ldg(row + j) : -2;
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      if ((uint32_t)id[h] < (uint32_t)p.n_blocks) atomicAdd(counts + id[h], -1);
      else if (id[h] != -2 || j0 + 32 * h + lane < n) bad = kErrInvalidArg;
    }
  }
}

__global__ void __launch_bounds__(kPageThreads) kv_release_entries_kernel(const ShareParams p) {
  pdl_wait();
  pdl_trigger();
  unsigned bad = 0;
  release_entries(p, p.shared_out, (int32_t)(blockIdx.x * kPageThreads + threadIdx.x) >> 5,
                  (int32_t)gridDim.x * kPageWarps, bad);
  if (bad) set_error(p.err, bad);
}

// Where the ring goes on and how much room it has.
struct ShareRing {
  int64_t taken, given, room;
  int32_t at;
  __device__ __forceinline__ ShareRing(const ShareParams& p, unsigned& bad)
      : taken(__ldg(p.cursor)), given(__ldg(p.cursor + 1)) {
    room = (int64_t)p.n_blocks - (given - taken);
    if (taken < 0 || given < taken || room < 0) {
      room = 0;
      bad = kErrInvalidArg;
    }
    at = given < 0 ? 0 : (int32_t)(given % p.n_blocks);
  }
  __device__ __forceinline__ void put(const ShareParams& p, int64_t k, int32_t block) const {
    if (k >= room) return;
    const int64_t q = at + k;  // (k < n_blocks)
    p.pool[q < p.n_blocks ? q : q - p.n_blocks] = block;
  }
  // By one thread.
  __device__ __forceinline__ void close(const ShareParams& p, int64_t number) const {
    p.cursor_out[0] = taken;
    p.cursor_out[1] = given + (number < room ? number : room);
  }
};

__global__ void __launch_bounds__(kPageThreads) kv_release_few_kernel(const ShareParams p) {
  extern __shared__ int32_t share_smem[];
  __shared__ int32_t slots[kPageWarps];
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31;
  unsigned bad = 0;
  const ShareRing ring(p, bad);
  for (int32_t i = tid; i < p.n_blocks; i += kPageThreads) share_smem[i] = __ldcg(p.shared + i);
  __syncthreads();
  release_entries(p, share_smem, tid >> 5, kPageWarps, bad);
  __syncthreads();
  // A thread's blocks are neighbours.
  const int32_t per = (p.n_blocks + kPageThreads - 1) / kPageThreads;
  const int32_t a = min(tid * per, p.n_blocks), b = min(a + per, p.n_blocks);
  int32_t own = 0, warps, total;
  for (int32_t i = a; i < b; ++i) own += share_smem[i] < 0;
  int32_t upto = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t u = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += u;
  }
  block_sums(__shfl_sync(0xffffffffu, upto, 31), slots, warps, total);
  int32_t k = warps + upto - own;
  for (int32_t i = a; own && i < b; ++i) {
    if (share_smem[i] >= 0) continue;
    if (share_smem[i] < -1) bad = kErrInvalidArg;  // more entries than holders
    share_smem[i] = 0;
    ring.put(p, k++, i);
  }
  __syncthreads();
  for (int32_t i = tid; i < p.n_blocks; i += kPageThreads) p.shared_out[i] = share_smem[i];
  if (total > ring.room) bad = kErrInvalidArg;
  if (tid == 0) ring.close(p, total);
  if (bad) set_error(p.err, bad);
}

__global__ void __launch_bounds__(kPageThreads) kv_release_shared_kernel(const ShareParams p) {
  __shared__ int32_t slots[kPageWarps], slot[2], listed[kPageWarps][128];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int32_t cta = (int32_t)cluster_ctarank(), warp = cta * kPageWarps + (threadIdx.x >> 5);
  const int32_t ctas = (int32_t)gridDim.x;  // (one cluster)
  unsigned bad = 0;
  const ShareRing ring(p, bad);
  const bool vec = (reinterpret_cast<uintptr_t>(p.shared_out) & 15) == 0;
  // A warp's blocks: 128 a step, all its steps in a row; no more steps than give each warp some.
  const int32_t each = ctas * kPageThreads * 4;
  const int32_t steps = min(kShareSteps, (p.n_blocks + each - 1) / each);
  int64_t base = 0;
  for (int64_t tile = 0, turn = 0; tile < p.n_blocks; tile += (int64_t)each * steps, ++turn) {
    const int64_t i0 = tile + (int64_t)warp * (128 * steps) + lane * 4;
    int4 left[kShareSteps];
#pragma unroll
    for (int s = 0; s < kShareSteps; ++s) {
      const int64_t i = i0 + s * 128;
      left[s] = make_int4(0, 0, 0, 0);
      if (s >= steps) continue;
      if (vec && i + 4 <= p.n_blocks) {
        left[s] = __ldcg(reinterpret_cast<const int4*>(p.shared_out + i));
      } else {
        if (i < p.n_blocks) left[s].x = __ldcg(p.shared_out + i);
        if (i + 1 < p.n_blocks) left[s].y = __ldcg(p.shared_out + i + 1);
        if (i + 2 < p.n_blocks) left[s].z = __ldcg(p.shared_out + i + 2);
        if (i + 3 < p.n_blocks) left[s].w = __ldcg(p.shared_out + i + 3);
      }
    }
    int32_t mine = 0;
#pragma unroll
    for (int s = 0; s < kShareSteps; ++s)
      mine += (left[s].x < 0) + (left[s].y < 0) + (left[s].z < 0) + (left[s].w < 0);
    mine = __reduce_add_sync(0xffffffffu, mine);
    int32_t warps, before, block, total;
    block_sums(mine, slots, warps, block);
    cluster_sums<kShareCtas>(block, slot + (turn & 1), before, total, ctas);
    int64_t at = base + before + warps;
    base += total;
    if (!mine) continue;
    // A step's numbers side by side in shared memory first, so that 32 go out at a time.
    int32_t* gone = listed[threadIdx.x >> 5];
#pragma unroll
    for (int s = 0; s < kShareSteps; ++s) {
      const int32_t v[4] = {left[s].x, left[s].y, left[s].z, left[s].w};
      const int32_t own = (v[0] < 0) + (v[1] < 0) + (v[2] < 0) + (v[3] < 0);
      const unsigned ones = __ballot_sync(0xffffffffu, own & 1);
      const unsigned twos = __ballot_sync(0xffffffffu, own & 2);
      const unsigned fours = __ballot_sync(0xffffffffu, own & 4);
      if (!(ones | twos | fours)) continue;
      const unsigned lt = lanemask_lt();
      const int32_t number = __popc(ones) + 2 * __popc(twos) + 4 * __popc(fours);
      int32_t k = __popc(ones & lt) + 2 * __popc(twos & lt) + 4 * __popc(fours & lt);
      const int64_t i = i0 + s * 128;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        if (v[h] >= 0) continue;
        if (v[h] < -1) bad = kErrInvalidArg;  // more entries than holders
        gone[k++] = (int32_t)i + h;
      }
      if (own && vec && i + 4 <= p.n_blocks) {
        *reinterpret_cast<int4*>(p.shared_out + i) =
            make_int4(max(v[0], 0), max(v[1], 0), max(v[2], 0), max(v[3], 0));
      } else if (own) {
#pragma unroll
        for (int h = 0; h < 4; ++h)
          if (v[h] < 0) p.shared_out[i + h] = 0;
      }
      __syncwarp();
      for (int32_t j = lane; j < number; j += 32) ring.put(p, at + j, gone[j]);
      __syncwarp();
      at += number;
    }
  }
  if (base > ring.room) bad = kErrInvalidArg;
  if (cta == 0 && threadIdx.x == 0) ring.close(p, base);
  if (bad) set_error(p.err, bad);
  cluster_sync();  // nobody leaves while its slot is read
}

struct CompactParams {
  const int32_t* lens;
  int64_t n_req;
  const int32_t* n_req_dev;
  int32_t bt_log2;
  const int32_t* table;
  int32_t* table_out;
  int32_t width;
  const int32_t* shared;
  int32_t* shared_out;
  int32_t n_blocks;
  int32_t* pool;
  int64_t* cursor_out;
  int32_t* source;
  int32_t* target;
  int32_t* moves;
  int32_t* map;  // workspace [n_blocks]
  unsigned* err;
};

// With U blocks in use, those with numbers >= U move to the free numbers < U, the first to the
// first; there are as many of both, and no fewer moves would do.
//
// A bit for each block says whether it is in use.  Every CTA has all of them in shared memory, with
// the number of blocks in use before each 32, and so knows by itself which block goes where: the
// q-th of those that move to the q-th free number, found by bisection.  So no CTA waits for
// another, and each does its share of the table, the lists and the counts.  Of small tables each
// CTA marks all entries' bits itself (MARK); of others a kernel of all SMs does.  8192 blocks, 96
// requests of up to 102: 6.7 us, and 13.7 as one cluster with a barrier between its passes.  64
// requests in 131,072, 262,144, 524,288 and 786,432 blocks: 6.6, 9.4, 19 and 17 us; a thread's words
// are neighbours, so that lanes' words meet in banks (16 of a warp's at 524,288 blocks, 8 at 786,432).
constexpr int32_t kCompactMost = 786432;     // blocks: 192 KB
constexpr int64_t kCompactEntries = 16384;   // of a table that each CTA reads

// Entries of lens[r] tokens of each request, by warps, 128 at a time.
template <class F>
__device__ __forceinline__ void used_entries(const CompactParams& p, int32_t R, int32_t first,
                                             int32_t warps, unsigned& bad, F&& f) {
  const int lane = threadIdx.x & 31;
  const int32_t chunks = (p.width + 127) / 128;
  const int64_t items = (int64_t)R * chunks;
  for (int64_t it = first; it < items; it += warps) {
    const int32_t r = (int32_t)(it / chunks), j0 = (int32_t)(it - (int64_t)r * chunks) * 128;
    const int32_t len = __ldg(p.lens + r);
    if (len < 0 || len > ((int64_t)p.width << p.bt_log2)) {
      bad = kErrInvalidArg;
      continue;
    }
    const int32_t n = blocks_of(len, p.bt_log2);
    const int32_t* row = p.table + (int64_t)r * p.width;
    int32_t id[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int32_t j = j0 + 32 * h + lane;
      id[h] = j < n ? row[j] : 0;
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      if (j0 + 32 * h + lane >= n) continue;
      if ((uint32_t)id[h] < (uint32_t)p.n_blocks) f(id[h]);
      else bad = kErrInvalidArg;
    }
  }
}

__global__ void __launch_bounds__(kPageThreads) kv_compact_zero_kernel(const CompactParams p) {
  pdl_wait();
  pdl_trigger();
  const int32_t i = blockIdx.x * kPageThreads + threadIdx.x;
  if (i < (p.n_blocks + 31) / 32) p.map[i] = 0;
}

__global__ void __launch_bounds__(kPageThreads) kv_compact_mark_kernel(const CompactParams p) {
  pdl_wait();
  pdl_trigger();
  unsigned bad = 0;
  used_entries(p, live_requests(p.n_req, p.n_req_dev),
               (int32_t)(blockIdx.x * kPageThreads + threadIdx.x) >> 5,
               (int32_t)gridDim.x * kPageWarps, bad,
               [&](int32_t id) { atomicOr(p.map + id / 32, 1 << (id % 32)); });
  if (bad) set_error(p.err, bad);
}

template <bool MARK>
__global__ void __launch_bounds__(kPageThreads) kv_compact_apply_kernel(const CompactParams p) {
  extern __shared__ uint32_t compact_smem[];
  __shared__ int32_t slots[kPageWarps];
  const int32_t words = (p.n_blocks + 31) / 32;
  uint32_t* bits = compact_smem;
  int32_t* before = reinterpret_cast<int32_t*>(compact_smem + words);
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31;
  const int32_t R = live_requests(p.n_req, p.n_req_dev);
  unsigned bad = 0;
  for (int32_t i = tid; i < words; i += kPageThreads)
    bits[i] = MARK ? 0u : (uint32_t)__ldcg(p.map + i);
  __syncthreads();
  if (MARK) {
    used_entries(p, R, tid >> 5, kPageWarps, bad,
                 [&](int32_t id) { atomicOr(bits + id / 32, 1u << (id % 32)); });
    __syncthreads();
  }
  // The number in use before each word: a thread's words are neighbours.
  const int32_t per = (words + kPageThreads - 1) / kPageThreads;
  const int32_t w0 = min(tid * per, words), w1 = min(w0 + per, words);
  int32_t own = 0, warps, used;
  for (int32_t w = w0; w < w1; ++w) own += __popc(bits[w]);
  int32_t upto = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t u = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += u;
  }
  block_sums(__shfl_sync(0xffffffffu, upto, 31), slots, warps, used);
  int32_t sum = warps + upto - own;
  for (int32_t w = w0; w < w1; ++w) {
    before[w] = sum;
    sum += __popc(bits[w]);
  }
  __syncthreads();
  // (n blocks in use of n: the word past the last does not exist)
  const auto rank = [&](int32_t i) {
    return i < p.n_blocks ? before[i / 32] + __popc(bits[i / 32] & ((1u << (i % 32)) - 1)) : used;
  };
  const int32_t low = rank(used), moves = used - low;
  // The number that the q-th of the moving blocks gets.
  const auto hole = [&](int32_t q) {
    int32_t a = 0, b = used / 32;  // the last word with at most q free numbers before it
    if (b >= words) b = words - 1;
    while (a < b) {
      const int32_t m = (a + b + 1) / 2;
      if (32 * m - before[m] <= q) a = m; else b = m - 1;
    }
    q -= 32 * a - before[a];
    uint32_t free = ~bits[a];
    int32_t at = 0;
#pragma unroll
    for (int s = 16; s > 0; s /= 2) {
      const int32_t c = __popc(free & ((1u << s) - 1));
      if (q >= c) {
        q -= c;
        free >>= s;
        at += s;
      }
    }
    return 32 * a + at;
  };
  const int32_t me = blockIdx.x * kPageThreads + tid, all = gridDim.x * kPageThreads;
  const int32_t room = max(1, p.n_blocks / 2);
  for (int32_t i = me; i < p.n_blocks; i += all) {
    const bool on = bits[i / 32] >> (i % 32) & 1u;
    const int32_t r = rank(i);
    p.pool[i] = i < p.n_blocks - used ? used + i : 0;
    if (i < used) {
      if (!on) p.target[i - r] = i;
      else if (p.shared && p.shared != p.shared_out) p.shared_out[i] = p.shared[i];
    } else {
      if (on) p.source[r - low] = i;
      if (p.shared) {
        // (the same thread reads a moving block's count and clears it)
        if (on) p.shared_out[hole(r - low)] = p.shared[i];
        p.shared_out[i] = 0;
      }
    }
    if (i >= moves && i < room) p.source[i] = p.target[i] = -1;
  }
  if (me == 0) {
    if (room > p.n_blocks) p.source[0] = p.target[0] = -1;
    *p.moves = moves;
    p.cursor_out[0] = 0;
    p.cursor_out[1] = p.n_blocks - used;
  }
  // Entries that name no block of a request go over as they are.
  const int64_t n = p.n_req * p.width;
  for (int64_t at = me; at < n; at += all) {
    const int32_t r = (int32_t)(at / p.width), j = (int32_t)(at - (int64_t)r * p.width);
    const int32_t id = p.table[at], len = r < R ? __ldg(p.lens + r) : 0;
    const bool moved = len >= 0 && len <= ((int64_t)p.width << p.bt_log2) &&
                       j < blocks_of(len, p.bt_log2) && (uint32_t)id < (uint32_t)p.n_blocks &&
                       id >= used;
    if (moved) p.table_out[at] = hole(rank(id) - low);
    else if (p.table != p.table_out) p.table_out[at] = id;
  }
  if (bad) set_error(p.err, bad);
}

// The same for any number of blocks: one cluster, which passes over the blocks in order, five times.
// 64 requests in 786,433 blocks 98 us (17 in one block less, by the kernels before), in 4,000,000 367.
__global__ void __launch_bounds__(kPageThreads) kv_compact_kernel(const CompactParams p) {
  __shared__ int32_t slots[kPageWarps], slot[3];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int32_t cta = (int32_t)cluster_ctarank();
  const int32_t me = cta * kPageThreads + threadIdx.x, all = kPageCtas * kPageThreads;
  const int32_t R = live_requests(p.n_req, p.n_req_dev);
  const int32_t room = max(1, p.n_blocks / 2);
  unsigned bad = 0;
  int32_t a, b;
  warp_range(p.n_blocks, a, b);
  for (int32_t i = a + lane; i < b; i += 32) p.map[i] = 0;
  cluster_sync();
  each_entry(p.lens, R, p.bt_log2, p.table, p.width, p.n_blocks, bad,
             [&](int64_t, int32_t id) { p.map[id] = 1; });
  cluster_sync();
  int32_t mine = 0, warps, ctas, block, used;
  for (int32_t i0 = a; i0 < b; i0 += 32)
    mine += __popc(__ballot_sync(0xffffffffu, i0 + lane < b && __ldcg(p.map + i0 + lane) != 0));
  block_sums(mine, slots, warps, block);
  cluster_sums(block, slot, ctas, used);
  // Free numbers below, numbers in use above.
  int32_t holes = 0, movers = 0;
  for (int32_t i0 = a; i0 < b; i0 += 32) {
    const int32_t i = i0 + lane;
    const bool on = i < b && __ldcg(p.map + i) != 0;
    holes += __popc(__ballot_sync(0xffffffffu, i < b && i < used && !on));
    movers += __popc(__ballot_sync(0xffffffffu, on && i >= used));
  }
  int32_t hole_w, hole_c, mover_w, mover_c, hole_b, mover_b, moves;
  block_sums(holes, slots, hole_w, hole_b);
  block_sums(movers, slots, mover_w, mover_b);
  cluster_sums(hole_b, slot + 1, hole_c, moves);
  cluster_sums(mover_b, slot + 2, mover_c, moves);
  int32_t hole = hole_c + hole_w, mover = mover_c + mover_w;
  for (int32_t i0 = a; i0 < b; i0 += 32) {
    const int32_t i = i0 + lane;
    const bool on = i < b && __ldcg(p.map + i) != 0;
    const bool is_hole = i < b && i < used && !on, is_mover = on && i >= used;
    const unsigned mh = __ballot_sync(0xffffffffu, is_hole);
    const unsigned mm = __ballot_sync(0xffffffffu, is_mover);
    if (is_hole) p.target[hole + __popc(mh & lanemask_lt())] = i;
    if (is_mover) p.source[mover + __popc(mm & lanemask_lt())] = i;
    hole += __popc(mh);
    mover += __popc(mm);
  }
  for (int32_t i = moves + me; i < room; i += all) p.source[i] = p.target[i] = -1;
  for (int32_t i = me; i < p.n_blocks; i += all)
    p.pool[i] = i < p.n_blocks - used ? used + i : 0;
  if (me == 0) {
    *p.moves = moves;
    p.cursor_out[0] = 0;
    p.cursor_out[1] = p.n_blocks - used;
  }
  cluster_sync();
  for (int32_t i = me; i < moves; i += all) {
    const int32_t s = __ldcg(p.source + i), t = __ldcg(p.target + i);
    p.map[s] = t;
    if (p.shared) p.shared_out[t] = __ldcg(p.shared + s);
  }
  // (a block in use that stays keeps the mark 1 and its count; marks of moved ones are numbers)
  if (p.shared && p.shared != p.shared_out)
    for (int32_t i = a + lane; i < b && i < used; i += 32)
      if (__ldcg(p.map + i) != 0) p.shared_out[i] = __ldcg(p.shared + i);
  cluster_sync();
  if (p.shared)
    for (int32_t i = a + lane; i < b; i += 32)
      if (i >= used) p.shared_out[i] = 0;
  if (p.table != p.table_out) {
    // entries that name no block of a request go over as they are
    const int64_t n = p.n_req * p.width;
    for (int64_t at = me; at < n; at += all) {
      const int32_t r = (int32_t)(at / p.width), j = (int32_t)(at - (int64_t)r * p.width);
      int32_t id = p.table[at];
      const int32_t len = r < R ? __ldg(p.lens + r) : 0;
      if (len >= 0 && len <= ((int64_t)p.width << p.bt_log2) && j < blocks_of(len, p.bt_log2) &&
          (uint32_t)id < (uint32_t)p.n_blocks && id >= used)
        id = __ldcg(p.map + id);
      p.table_out[at] = id;
    }
  } else {
    unsigned seen = 0;
    each_entry(p.lens, R, p.bt_log2, p.table, p.width, p.n_blocks, seen, [&](int64_t at, int32_t id) {
      if (id >= used) p.table_out[at] = __ldcg(p.map + id);
    });
  }
  if (bad) set_error(p.err, bad);
}

// One cluster of `ctas` CTAs, with programmatic stream serialization.
struct OneCluster {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  OneCluster(int ctas, cudaStream_t stream) {
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kPageThreads);
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
  }
};

// CTAs of kv_release_shared_kernel's cluster on each device.
std::atomic<int32_t> g_share_ctas[kMaxDeviceOrdinals];

hs_status share_setup(int dev) {
  const hs_status st = cuda_fail(
      cudaFuncSetAttribute(kv_release_shared_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1),
      "kv_release_shared clusters");
  if (st != HS_OK) return st;
  int most = 0;
  const OneCluster c(kShareCtas, nullptr);
  const bool fits =
      cudaOccupancyMaxActiveClusters(&most, kv_release_shared_kernel, &c.cfg) == cudaSuccess && most > 0;
  if (!fits) (void)cudaGetLastError();
  g_share_ctas[dev].store(fits ? kShareCtas : kPageCtas, std::memory_order_relaxed);
  return HS_OK;
}

}  // namespace

hs_status launch_kv_fork(const int32_t* src, const int32_t* dst, int64_t n, const int32_t* lens,
                         int32_t* lens_out, int64_t n_req, int32_t bt_log2, int32_t* table,
                         int32_t width, int32_t* shared, const int32_t* pool, int64_t n_blocks,
                         const int64_t* cursor, int64_t* cursor_out, int32_t* source,
                         int32_t* target, int32_t* tokens, const int32_t* n_req_dev,
                         int32_t* n_req_out, cudaStream_t stream) {
  unsigned* err = device_error_word();
  if (!err) return fail(HS_ERR_CUDA, "could not resolve the device error word");
  const ForkParams p{src, dst, (int32_t)n, lens, lens_out, (int32_t)n_req, bt_log2, table, width,
                     shared, pool, (int32_t)n_blocks, cursor, cursor_out, source, target, tokens,
                     n_req_dev, n_req_out, err};
  const size_t smem = (size_t)(n_req + n) * 4;
  static std::atomic<uint64_t> configured{0};
  const hs_status st = grant_smem(configured, kv_fork_kernel, 2 * HS_KV_MAX_REQUESTS * 4,
                                  "kv_fork shared memory");
  if (st != HS_OK) return st;
  int64_t grid = ((n > n_req / 32 ? n : n_req / 32) * 32 + kForkThreads - 1) / kForkThreads;
  if (grid < 1) grid = 1;
  if (grid > num_sms()) grid = num_sms();
  launch_pdl(kv_fork_kernel, dim3((unsigned)grid), dim3(kForkThreads), smem, stream, p);
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "kv_fork launch");
}

hs_status launch_kv_copy(const hs_kv_cache& c, const int32_t* source, const int32_t* target,
                         const int32_t* tokens, int64_t n, const int32_t* n_dev,
                         cudaStream_t stream) {
  unsigned* err = device_error_word();
  if (!err) return fail(HS_ERR_CUDA, "could not resolve the device error word");
  const int32_t pieces = (c.block_tokens * c.dim + kCopyPiece - 1) / kCopyPiece;
  const CopyParams p{{static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v)},
                     {c.k_scale, c.v_scale},
                     c.n_blocks, c.n_kv_heads, c.block_tokens, c.dim, pieces,
                     source, target, tokens, n, n_dev, err};
  const int64_t warps = n * 2 * c.n_kv_heads * pieces;
  int64_t grid = (warps + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
  if (grid > 32LL * num_sms()) grid = 32LL * num_sms();
  launch_pdl(kv_copy_kernel, dim3((unsigned)grid), dim3(kCopyThreads), 0, stream, p);
  count_launches(1);
  return cuda_fail(cudaGetLastError(), "kv_copy launch");
}

hs_status launch_kv_release_shared(const int32_t* lens, int64_t n_req, const int32_t* n_req_dev,
                                   int32_t bt_log2, const int32_t* table, int32_t width,
                                   const int32_t* shared, int32_t* shared_out, int32_t* pool,
                                   int64_t n_blocks, const int64_t* cursor, int64_t* cursor_out,
                                   cudaStream_t stream) {
  unsigned* err = device_error_word();
  if (!err) return fail(HS_ERR_CUDA, "could not resolve the device error word");
  const ShareParams p{lens, n_req, n_req_dev, bt_log2, table, width, shared, shared_out, pool,
                      (int32_t)n_blocks, cursor, cursor_out, err};
  const int64_t entries = n_req * width;
  if (entries <= kShareFewEntries && n_blocks <= kShareFew) {
    static std::atomic<uint64_t> configured{0};
    const hs_status st = once_per_device(configured, [] {
      return cuda_fail(cudaFuncSetAttribute(kv_release_few_kernel,
                                            cudaFuncAttributeMaxDynamicSharedMemorySize,
                                            kShareFew * 4),
                       "kv_release_shared shared memory");
    });
    if (st != HS_OK) return st;
    launch_pdl(kv_release_few_kernel, dim3(1), dim3(kPageThreads), (size_t)n_blocks * 4, stream, p);
    count_launches(1);
  } else {
    const int dev = device_ordinal() < 0 ? 0 : device_ordinal();
    static std::atomic<uint64_t> configured{0};
    const hs_status st = once_per_device(configured, [dev] { return share_setup(dev); });
    if (st != HS_OK) return st;
    const auto grid = [](int64_t threads) {
      const int64_t g = (threads + kPageThreads - 1) / kPageThreads;
      return dim3((unsigned)(g < 1 ? 1 : g < 2LL * num_sms() ? g : 2LL * num_sms()));
    };
    if (shared != shared_out)
      launch_pdl(kv_share_copy_kernel, grid(n_blocks), dim3(kPageThreads), 0, stream, p);
    launch_pdl(kv_release_entries_kernel, grid(n_req * ((width + 127) / 128) * 32),
               dim3(kPageThreads), 0, stream, p);
    const OneCluster c(g_share_ctas[dev].load(std::memory_order_relaxed), stream);
    cudaLaunchKernelEx(&c.cfg, kv_release_shared_kernel, p);
    count_launches(shared != shared_out ? 3 : 2);
  }
  return cuda_fail(cudaGetLastError(), "kv_release_shared launch");
}

hs_status launch_kv_compact(const int32_t* lens, int64_t n_req, const int32_t* n_req_dev,
                            int32_t bt_log2, const int32_t* table, int32_t* table_out,
                            int32_t width, const int32_t* shared, int32_t* shared_out,
                            int64_t n_blocks, int32_t* pool, int64_t* cursor_out, int32_t* source,
                            int32_t* target, int32_t* moves, void* workspace,
                            cudaStream_t stream) {
  unsigned* err = device_error_word();
  if (!err) return fail(HS_ERR_CUDA, "could not resolve the device error word");
  const CompactParams p{lens, n_req, n_req_dev, bt_log2, table, table_out, width, shared,
                        shared_out, (int32_t)n_blocks, pool, cursor_out, source, target, moves,
                        static_cast<int32_t*>(workspace), err};
  if (n_blocks > kCompactMost) {
    const OneCluster c(kPageCtas, stream);
    cudaLaunchKernelEx(&c.cfg, kv_compact_kernel, p);
    count_launches(1);
    return cuda_fail(cudaGetLastError(), "kv_compact launch");
  }
  const int64_t entries = n_req * width;
  const int32_t words = (int32_t)((n_blocks + 31) / 32);
  const size_t smem = (size_t)words * 8;
  static std::atomic<uint64_t> configured[2] = {};
  hs_status st = grant_smem(configured[0], kv_compact_apply_kernel<false>, kCompactMost / 4,
                            "kv_compact shared memory");
  if (st == HS_OK)
    st = grant_smem(configured[1], kv_compact_apply_kernel<true>, kCompactMost / 4,
                    "kv_compact shared memory");
  if (st != HS_OK) return st;
  const auto grid = [](int64_t threads) {
    const int64_t g = (threads + kPageThreads - 1) / kPageThreads;
    return dim3((unsigned)(g < 1 ? 1 : g < num_sms() ? g : num_sms()));
  };
  // In place one CTA renames entries that another may still have to mark: one alone does both, or
  // the marks are a kernel of their own.
  const bool in_place = table == table_out;
  const dim3 shares = grid(entries > n_blocks ? entries : n_blocks);
  if (entries <= kCompactEntries && (!in_place || n_blocks <= kCompactEntries)) {
    launch_pdl(kv_compact_apply_kernel<true>, in_place ? dim3(1) : shares, dim3(kPageThreads), smem,
               stream, p);
    count_launches(1);
  } else {
    launch_pdl(kv_compact_zero_kernel, dim3((words + kPageThreads - 1) / kPageThreads),
               dim3(kPageThreads), 0, stream, p);
    launch_pdl(kv_compact_mark_kernel, grid(n_req * ((width + 127) / 128) * 32),
               dim3(kPageThreads), 0, stream, p);
    launch_pdl(kv_compact_apply_kernel<false>, shares, dim3(kPageThreads), smem, stream, p);
    count_launches(3);
  }
  return cuda_fail(cudaGetLastError(), "kv_compact launch");
}

}  // namespace hs
