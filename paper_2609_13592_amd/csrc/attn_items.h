// Work items of the paged-attention decode: the parameters of a call, how the
// requests' contexts are cut into partitions, and how a workgroup finds its
// item; shared by the kernels of both pool formats.
#pragma once
#include "runtime.h"

namespace bst {
namespace attn {

constexpr int kThreads = 256;
constexpr int kD = 128;          // head dimension of these kernels
constexpr int kT = 16;           // tokens per block
// Work items a launch aims for (partition size follows; config 3: 2048
// items of 64 blocks ran 120 us against 122 us with 4096 of 32)
#ifndef BOOST_ATTN_ITEMS
#define BOOST_ATTN_ITEMS 2048
#endif
// A 4-bit item carries a quarter of the bytes, so fewer are aimed for (64
// requests of 512..4096: 36.5 us with 768, 37.5 with 1024, two of 100000 44.0
// and 45.5; with 2048 5 to 10 % more)
#ifndef BOOST_ATTN_ITEMS4
#define BOOST_ATTN_ITEMS4 768
#endif
// 4-bit contexts of up to this many blocks stay whole, a launch without a
// merge: where their workgroups leave half of the compute units empty (one
// request of 301 tokens 4.9 us, cut in five 7.2; of 1000 7.6 and 7.4), and
// where they do not (16 requests of 2000 tokens 12.7 and 14.5, of 4000 21.5 and
// 20.4; 64 of 2000 27.4 and 31.5).
constexpr int kOneFew = 60, kOneMany = 160;
constexpr int kMaxPartBlocks = 256;         // blocks per partition, at most
static_assert(kMaxPartBlocks <= kThreads, "one thread per partition size");
// A work item of fewer than 16 blocks spends as long on its start (q loads)
// and end (slot merge, partial stores) as on its K/V (batch 8 at 2048 tokens:
// 1.2 TB/s with 4-block items, 2.2 TB/s with 16).
#ifndef BOOST_ATTN_PART_MIN
#define BOOST_ATTN_PART_MIN 16
#endif
#ifndef BOOST_ATTN_PART_MAX
#define BOOST_ATTN_PART_MAX 256
#endif
constexpr int kPartMin = BOOST_ATTN_PART_MIN, kPartMax = BOOST_ATTN_PART_MAX;
// ... but while such items are fewer than the compute units they are halved,
// down to four blocks: a longer chain of loads on some units is then worse
// than the starts and ends of more items (32 / 8 heads, one request of 500 /
// 2048 tokens: 16.6 / 17.1 -> 10.0 / 11.6 us, four of 200..1000: 16.8 -> 11.4;
// with enough items it loses, one of 8192: 19.2 -> 20.7).  The items are
// counted from the width of the block table, since the host does not know the
// context lengths: short contexts in a wide table keep kPartMin.
constexpr int kPartFew = 4;

struct AttnParams {
  // Linear placement makes the tier of a pool page a fixed function of its
  // offset: pages [0, first_host) of a tensor are consecutive in the HBM slab
  // and pages [first_host, pages) consecutive in the host slab.
  const char* k_hbm;   // this layer's K tensor: first HBM page
  const char* k_host;  // ... first host page
  const char* v_hbm;
  const char* v_host;
  uint64_t host_from;  // byte offset where the tensor's host tail begins
  const uint16_t* q;      // [B, Hq, D]
  const int32_t* tables;  // [B, max_blocks]
  const int32_t* lens;    // [B]
  int B, H, Hq, nb, max_blocks;
  // attention over selected blocks: per request and KV head the list
  // [top_k] of block indices of the context (null: every block)
  const int32_t* sel;
  int top_k;
  int item_blocks;  // blocks of a request that count, at most: max_blocks, with a list min(max_blocks, top_k)
  int part_blocks, n_parts;  // partition size in blocks, partitions per request
  int max_parts;             // stride of the partial buffers
  float scale;
  float* part_acc;  // [B * Hq * max_parts][D] unnormalised sums of p * v
  float* part_ml;   // [B * Hq * max_parts][2] running max of q . k, sum of p
  void* out;
  int out_bf16;
  int one_done;  // contexts of one partition are finished without the merge
};

__device__ __forceinline__ uint16_t to_bf16(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7f800000u) == 0x7f800000u && (u & 0x007fffffu)) return 0x7fc0;
  u += 0x7fffu + ((u >> 16) & 1u);
  return static_cast<uint16_t>(u >> 16);
}

// Blocks of L > 0 tokens (any: L + 15 need not fit).
__device__ __forceinline__ int blocks_in(int L) { return (L - 1) / kT + 1; }

// Blocks of request b in this call (0 for an empty context).
__device__ __forceinline__ int blocks_of(const AttnParams& P, int b) {
  const int L = P.lens[b];
  return L <= 0 ? 0 : min(blocks_in(L), P.item_blocks);
}

// Sum of v over the workgroup; every thread gets it (red: 4 ints of LDS).
__device__ __forceinline__ int wg_sum(int v, int* red) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
  __syncthreads();  // red is free again
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}

// Exclusive prefix sum of v over the workgroup in thread order; total gets
// the sum of every thread's v.
__device__ __forceinline__ int wg_scan(int v, int* red, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) red[wave] = x;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += red[w];
  total = red[0] + red[1] + red[2] + red[3];
  return before + x - v;
}

// Request whose count interval holds `target` in the running sum of
// count(n_b) over b = 0, 1, ... (count > 0 there); pick[0] gets b, pick[1]
// target minus the sum before b, pick[4] b's context length.  n0, L0: this
// thread's n_b and length for b = threadIdx.x (read once by the caller);
// later chunks read the lengths again.
template <typename Count>
__device__ __forceinline__ void find_request(const AttnParams& P, int target, int n0, int L0,
                                             Count count, int* red, int* pick) {
  int carry = 0;
  for (int base = 0; base < P.B; base += kThreads) {  // uniform
    const int b = base + static_cast<int>(threadIdx.x);
    const int c = b < P.B ? count(base == 0 ? n0 : blocks_of(P, b)) : 0;
    int total;
    const int ex = carry + wg_scan(c, red, total);
    if (c > 0 && ex <= target && target < ex + c) {
      pick[0] = b;
      pick[1] = target - ex;
      pick[4] = base == 0 ? L0 : P.lens[b];
    }
    carry += total;
    if (carry > target) break;  // uniform
  }
  __syncthreads();
}

// The item of item_of (below) for at most 64 requests: one request per lane,
// every wavefront by itself, with ballots instead of barriers (0.9 us less
// before an item's first loads).
__device__ __forceinline__ bool item_of_wave(const AttnParams& P, int idx, int& b, int& g,
                                             int& part, int& L) {
  const int lane = threadIdx.x & 63, PB = P.part_blocks, H = P.H;
  const int L0 = lane < P.B ? P.lens[lane] : 0;
  const int n = L0 <= 0 ? 0 : min(blocks_in(L0), P.item_blocks);
  const int full = n / PB, rem = n % PB;
  // inclusive prefix sums of both counts over the requests
  int xf = full, xr = rem > 0;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int yf = __shfl_up(xf, d, 64), yr = __shfl_up(xr, d, 64);
    if (lane >= d) {
      xf += yf;
      xr += yr;
    }
  }
  const int F = __builtin_amdgcn_readlane(xf, 63), R = __builtin_amdgcn_readlane(xr, 63);
  auto pick = [&](unsigned long long who) {
    b = __builtin_amdgcn_readfirstlane(static_cast<int>(__ffsll(who)) - 1);
    L = __builtin_amdgcn_readlane(L0, b);
  };
  if (idx < F + R) {  // every partition of head H-1
    const int end = xf + xr, beg = end - full - (rem > 0);
    const unsigned long long who = __ballot(beg <= idx && idx < end);
    if (!who) return false;
    pick(who);
    part = idx - __builtin_amdgcn_readlane(beg, b);
    g = H - 1;
    return true;
  }
  int j = idx - (F + R);
  if (j < (H - 1) * F) {  // full partitions of the others
    const int t = j / (H - 1);
    const unsigned long long who = __ballot(xf - full <= t && t < xf);
    if (!who) return false;
    pick(who);
    part = t - __builtin_amdgcn_readlane(xf - full, b);
    g = H - 2 - j % (H - 1);
    return true;
  }
  j -= (H - 1) * F;
  if (j >= (H - 1) * R) return false;
  // partial partitions by size: the rank-th largest rem (below 256), bit by
  // bit, then the requests of that size in order
  int rank = j / (H - 1);
  unsigned long long who = __ballot(rem > 0);
#pragma unroll
  for (int bit = 7; bit >= 0; --bit) {
    const unsigned long long ones = who & __ballot(rem >> bit & 1);
    const int c = __popcll(ones);
    if (rank < c) {
      who = ones;
    } else {
      rank -= c;
      who &= ~ones;
    }
  }
  const int before = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(who >> 32),
                                               __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(who), 0));
  const unsigned long long one = __ballot((who >> lane & 1) && before == rank);
  if (!one) return false;
  pick(one);
  part = __builtin_amdgcn_readlane(full, b);
  g = H - 2 - j % (H - 1);
  return true;
}

// Work item of workgroup idx, from the context lengths alone (so the same on
// every pool: the order decides which items run together, never what an item
// computes).  With n_b blocks, request b has full_b = n_b / part_blocks full
// partitions and one partial one if rem_b = n_b % part_blocks > 0.  Order:
//   1. every partition of head H-1 (where host data can lie), request by
//      request: its slow reads start first;
//   2. full partitions of heads H-2..0, request by request, head fastest;
//   3. partial partitions of heads H-2..0, the largest first (rem_b
//      descending, then b ascending), head fastest;
//   4. workgroups past the last item return at once.
// Empty partitions get no workgroup and the short ones run last, so the last
// grid wave is short (config 3, reads alone: 104 -> 96 us).
// L gets the request's context length (so the caller does not read it again).
__device__ inline bool item_of(const AttnParams& P, int idx, int& b, int& g, int& part, int& L,
                        int* red, int* hist, int* pick) {
  const int tid = threadIdx.x, PB = P.part_blocks, H = P.H;
  if (tid < 5) pick[tid] = -1;  // written by the sums' barriers below
  const int L0 = tid < P.B ? P.lens[tid] : 0;  // request tid, read once
  const int n0 = L0 <= 0 ? 0 : min(blocks_in(L0), P.item_blocks);
  int f = 0, r = 0;
  for (int bb = tid; bb < P.B; bb += kThreads) {
    const int n = bb == tid ? n0 : blocks_of(P, bb);
    f += n / PB;
    r += n % PB > 0;
  }
  const int F = wg_sum(f, red), R = wg_sum(r, red);
  const int S0 = F + R;
  if (idx < S0) {
    find_request(P, idx, n0, L0, [&](int n) { return n / PB + (n % PB > 0); }, red, pick);
    b = pick[0];
    part = pick[1];
    L = pick[4];
    g = H - 1;
    return b >= 0 && b < P.B && part >= 0;
  }
  int j = idx - S0;
  if (j < (H - 1) * F) {
    find_request(P, j / (H - 1), n0, L0, [&](int n) { return n / PB; }, red, pick);
    b = pick[0];
    part = pick[1];
    L = pick[4];
    g = H - 2 - j % (H - 1);
    return b >= 0 && b < P.B && part >= 0;
  }
  j -= (H - 1) * F;
  if (j >= (H - 1) * R) return false;
  // partial partitions by size: a counting sort over rem in [1, PB)
  const int rank = j / (H - 1);
  for (int v = tid; v < PB; v += kThreads) hist[v] = 0;
  __syncthreads();
  for (int bb = tid; bb < P.B; bb += kThreads) {
    const int rem = (bb == tid ? n0 : blocks_of(P, bb)) % PB;
    if (rem > 0) atomicAdd(&hist[rem], 1);
  }
  __syncthreads();
  {
    const int v = PB - 1 - tid;  // thread order = rem descending (PB <= kThreads)
    const int c = v >= 1 ? hist[v] : 0;
    int total;
    const int ex = wg_scan(c, red, total);
    if (c > 0 && ex <= rank && rank < ex + c) {
      pick[2] = v;
      pick[3] = rank - ex;
    }
    __syncthreads();
  }
  const int vsel = pick[2];
  find_request(P, pick[3], n0, L0, [&](int n) { return n % PB == vsel ? 1 : 0; }, red, pick);
  b = pick[0];
  if (b < 0 || b >= P.B) return false;
  L = pick[4];
  part = (L <= 0 ? 0 : min(blocks_in(L), P.item_blocks)) / PB;
  g = H - 2 - j % (H - 1);
  return true;
}

// Work item of a call over lists, or of one whose contexts have one partition:
// a grid of requests, KV heads and partitions, the empty ones too.  Nothing is
// read or divided for it, and lists differ little in length.
__device__ __forceinline__ void item_each(const AttnParams& P, int& b, int& g, int& part) {
  b = blockIdx.x;
  g = P.H - 1 - static_cast<int>(blockIdx.y);
  part = blockIdx.z;
}
// (false: more than a grid holds)
inline bool grid_each(const AttnParams& P, dim3& grid) {
  grid = dim3(P.B, P.H, P.n_parts);
  return P.H <= 65535 && P.n_parts <= 65535;
}

// Entry i of partition `part` of the list of (request b, KV head g), past its
// end the last: its index in the context and the pool block there, loaded
// without waiting for the context's length (and by every thread: behind a branch
// on the thread the compiler took the partition for one of the thread's own).
struct Listed {
  int32_t at, block;
};
__device__ __forceinline__ Listed listed(const AttnParams& P, int b, int g, int part, int i) {
  const int k = min(part * P.part_blocks + min(i, P.part_blocks - 1), P.top_k - 1);
  const int32_t at = P.sel[(static_cast<int64_t>(b) * P.H + g) * P.top_k + k];
  return {at, P.tables[static_cast<int64_t>(b) * P.max_blocks + min(max(at, 0), P.max_blocks - 1)]};
}
// ... as a context of L tokens has it: -1 where the entry names no block of it
// (its tokens are left out); tok gets how many of its tokens lie inside.
__device__ __forceinline__ int32_t selected(const AttnParams& P, const Listed& e, int L, int32_t& tok) {
  const bool in = e.at >= 0 && e.at < P.max_blocks && e.at <= (L - 1) / kT;
  tok = in ? min(kT, L - e.at * kT) : 0;
  return in ? e.block : -1;
}

// The kernels of a 4-bit pool: launches the partitions (any Hq / H up to 8).
// Contexts of one partition are finished there; if none has more (n_parts 1),
// empty ones too, and there is nothing to merge.
int launch_fp4(AttnParams& P, int n_cu, hipStream_t s);

}  // namespace attn
}  // namespace bst
