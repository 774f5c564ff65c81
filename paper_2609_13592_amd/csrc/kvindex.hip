// Block summaries of a KV pool and the selection of blocks by them: what
// sparse attention reads in place of a long context.
//
// Summary of a head-block: for every dim the largest and the smallest key of
// its live tokens, outwards in whole steps of 2^e, e the smallest (>= -126)
// with max|k| <= 127 * 2^e:
//   hi_d = ceil(max_t k_td / 2^e)   lo_d = floor(min_t k_td / 2^e)   (int8)
// Score of a block for a query head: q8 = round(q / 2^eq) (the same rule for
// eq, ties to even, at most 127), 2^(e + eq) sum_d max(q8_d hi_d, q8_d lo_d),
// an upper bound of q8 . k over the block's tokens; for a KV head the largest
// over its query heads.  The sum is one of whole numbers below 2^21 and the
// factor a power of two, so a score is exact and a selection does not depend
// on the order of any sum: the same blocks on every placement, split and
// machine.  257 bytes stand for the 8 KiB (bf16) of a head-block.
#include <algorithm>
#include <cmath>

#include "kvfmt.h"
#include "runtime.h"

namespace {

constexpr int kD = 128;
constexpr int kT = 16;
constexpr int kSum = 2 * kD;      // bytes of a summary: hi, then lo
constexpr int kNotFinite = 127;   // exponent byte of a block with an inf or NaN key

typedef __attribute__((ext_vector_type(4))) int i32x4;

struct IndexParams {
  const char* const* pt_k;  // this layer's K pages
  int8_t* sum;              // this layer's summaries [H][nb][256]
  int8_t* exp;              // and exponents [H][nb]
  const int32_t* tables;    // [B, max_blocks]
  const int32_t* starts;    // [B] tokens [starts, ends) are new
  const int32_t* ends;
  int B, H, nb, max_blocks;
};

// e of the rule above for a largest magnitude given by its bf16 bits (below
// 0x7f80).  amax = 2^E (1 + m / 128) is at most 127 * 2^(E - 6) unless m = 127.
__device__ __forceinline__ int step_exponent(uint32_t amax) {
  const int f = static_cast<int>(amax >> 7);
  return f == 0 ? -126 : max(f - 133 + ((amax & 127) == 127), -126);
}
__device__ __forceinline__ float pow2f(int e) {  // -126 <= e <= 127
  return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}
__device__ __forceinline__ float lo_bf16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1)
    v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), m, 64)));
  return v;
}

// One wavefront per head-block.  FP4: lane (token r, group qd); else lane
// (8-dim chunk, token row qd of four).
template <bool FP4>
__global__ __launch_bounds__(256) void index_update_kernel(IndexParams P, int chunks) {
  const int lane = threadIdx.x & 63, r = lane & 15, qd = lane >> 4;
  const int chunk = blockIdx.x % chunks, bg = blockIdx.x / chunks;
  const int g = bg % P.H, b = bg / P.H;
  const int start = max(P.starts[b], 0);
  const int end = static_cast<int>(
      min(static_cast<int64_t>(P.ends[b]), static_cast<int64_t>(P.max_blocks) * kT));
  if (start >= end) return;
  const int last = (end - 1) / kT;
  for (int blk = start / kT + chunk * 4 + static_cast<int>(threadIdx.x >> 6); blk <= last;
       blk += chunks * 4) {
    const int32_t id = P.tables[static_cast<int64_t>(b) * P.max_blocks + blk];
    if (id < 0 || id >= P.nb) continue;  // uniform over the wavefront
    const int live = min(kT, end - blk * kT);
    const int64_t at = static_cast<int64_t>(g) * P.nb + id;
    int8_t* const out = P.sum + at * kSum;
    uint32_t amax = 0;  // bf16 bits
    if constexpr (FP4) {
      using namespace bst;
      const Fp4At f = fp4_at(g, id, P.nb);
      const char* const page = P.pt_k[f.page];
      const uint4 c = *reinterpret_cast<const uint4*>(page + f.idx * kFp4Code + r * 64 + qd * 16);
      const uint32_t sb = static_cast<uint8_t>(
          page[kFp4ScaleAt + f.idx * kFp4Scale + r * 4 + qd]);
      const bool in = r < live;
      const float s = fp4_scale(sb);
      float mx[32], mn[32];
      const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t p[4] = {fp4_unpack<0>(w[i], s), fp4_unpack<1>(w[i], s),
                               fp4_unpack<2>(w[i], s), fp4_unpack<3>(w[i], s)};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          amax = max(amax, max(p[j] & 0x7fffu, (p[j] >> 16) & 0x7fffu));
          mx[8 * i + 2 * j] = in ? lo_bf16(p[j]) : -INFINITY;
          mx[8 * i + 2 * j + 1] = in ? hi_bf16(p[j]) : -INFINITY;
          mn[8 * i + 2 * j] = in ? lo_bf16(p[j]) : INFINITY;
          mn[8 * i + 2 * j + 1] = in ? hi_bf16(p[j]) : INFINITY;
        }
      }
      amax = wave_max(in ? amax : 0);
      // over the 16 tokens, half of the dims kept in each step: lane r ends
      // with dims 2 r, 2 r + 1 of its group
#pragma unroll
      for (int n = 16, m = 8; m >= 1; n >>= 1, m >>= 1) {
        const bool up = lane & m;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (i >= n) break;
          const float keep_x = up ? mx[n + i] : mx[i], give_x = up ? mx[i] : mx[n + i];
          const float keep_n = up ? mn[n + i] : mn[i], give_n = up ? mn[i] : mn[n + i];
          mx[i] = fmaxf(keep_x, __shfl_xor(give_x, m, 64));
          mn[i] = fminf(keep_n, __shfl_xor(give_n, m, 64));
        }
      }
      const int e = amax >= 0x7f80 ? kNotFinite : step_exponent(amax);
      const float step = pow2f(e == kNotFinite ? 0 : -e);
      int8_t* const o = out + 32 * qd + 2 * r;
      const bool bad = e == kNotFinite;  // no numbers to keep
      *reinterpret_cast<char2*>(o) =
          bad ? char2{0, 0}
              : char2{static_cast<signed char>(ceilf(mx[0] * step)),
                      static_cast<signed char>(ceilf(mx[1] * step))};
      *reinterpret_cast<char2*>(o + kD) =
          bad ? char2{0, 0}
              : char2{static_cast<signed char>(floorf(mn[0] * step)),
                      static_cast<signed char>(floorf(mn[1] * step))};
      if (lane == 0) P.exp[at] = static_cast<int8_t>(e);
    } else {
      const uint64_t byte = static_cast<uint64_t>(at) * kT * kD * 2;
      const char* const src = P.pt_k[byte >> 21] + (byte & (bst::kPage - 1)) + r * 16;
      float mx[8], mn[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        mx[i] = -INFINITY;
        mn[i] = INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = 4 * i + qd;
        const uint4 u = *reinterpret_cast<const uint4*>(src + t * kD * 2);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        if (t < live) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            amax = max(amax, max(w[j] & 0x7fffu, (w[j] >> 16) & 0x7fffu));
            mx[2 * j] = fmaxf(mx[2 * j], lo_bf16(w[j]));
            mx[2 * j + 1] = fmaxf(mx[2 * j + 1], hi_bf16(w[j]));
            mn[2 * j] = fminf(mn[2 * j], lo_bf16(w[j]));
            mn[2 * j + 1] = fminf(mn[2 * j + 1], hi_bf16(w[j]));
          }
        }
      }
      amax = wave_max(amax);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        mx[i] = fmaxf(mx[i], __shfl_xor(mx[i], 16, 64));
        mx[i] = fmaxf(mx[i], __shfl_xor(mx[i], 32, 64));
        mn[i] = fminf(mn[i], __shfl_xor(mn[i], 16, 64));
        mn[i] = fminf(mn[i], __shfl_xor(mn[i], 32, 64));
      }
      const int e = amax >= 0x7f80 ? kNotFinite : step_exponent(amax);
      const float step = pow2f(e == kNotFinite ? 0 : -e);
      uint32_t w[2] = {0, 0};
      if (e != kNotFinite) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int v = static_cast<int>(qd == 0 ? ceilf(mx[i] * step) : floorf(mn[i] * step));
          w[i / 4] |= (static_cast<uint32_t>(v) & 255u) << (8 * (i % 4));
        }
      }
      if (qd < 2) *reinterpret_cast<uint2*>(out + qd * kD + r * 8) = make_uint2(w[0], w[1]);
      if (lane == 0) P.exp[at] = static_cast<int8_t>(e);
    }
  }
}

struct SelectParams {
  const int8_t* sum;
  const int8_t* exp;
  const uint16_t* q;      // [B, Hq, D]
  const int32_t* tables;  // [B, max_blocks]
  const int32_t* lens;    // [B]
  float* scores;          // [B, H, max_blocks]
  int32_t* sel;           // [B, H, top_k]
  int B, H, Hq, nb, max_blocks;
  int top_k, n_first, n_last;
};

__device__ __forceinline__ int context_blocks(const SelectParams& P, int b) {
  const int L = P.lens[b];
  return L <= 0 ? 0 : min((L - 1) / kT + 1, P.max_blocks);
}

// Scores of 16-block tiles, one wavefront a tile: rows are blocks, columns
// the KV head's query heads, the 256 products of a pair in four 16x16x64
// integer products (hi against the positive part of q8, lo against the
// negative).  Bound by the summaries' bytes.
constexpr int kTileBlocks = 16, kTilesPerWave = 4;
constexpr int kScoreBlocks = 4 * kTileBlocks * kTilesPerWave;  // per workgroup

__global__ __launch_bounds__(256) void block_scores_kernel(SelectParams P, int chunks) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, qd = lane >> 4;
  const int chunk = blockIdx.x % chunks, bg = blockIdx.x / chunks;
  const int g = bg % P.H, b = bg / P.H;
  const int n = context_blocks(P, b);
  if (chunk * kScoreBlocks >= n) return;  // uniform
  const int G = P.Hq / P.H;
  // column r: head r (zero beyond G), dims 16 qd .. + 15 and 64 more
  i32x4 qb[4];
  int eq;
  {
    const uint4* q = reinterpret_cast<const uint4*>(
        P.q + (static_cast<int64_t>(b) * P.Hq + g * G + min(r, G - 1)) * kD + 16 * qd);
    uint32_t w[16], amax = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 u = q[i < 2 ? i : 6 + i];  // 64 dims are 8 uint4 further
      w[4 * i] = u.x;
      w[4 * i + 1] = u.y;
      w[4 * i + 2] = u.z;
      w[4 * i + 3] = u.w;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) amax = max(amax, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
    amax = max(amax, static_cast<uint32_t>(__shfl_xor(static_cast<int>(amax), 16, 64)));
    amax = max(amax, static_cast<uint32_t>(__shfl_xor(static_cast<int>(amax), 32, 64)));
    const bool none = amax >= 0x7f80 || r >= G;  // a query that is not finite counts as 0
    eq = none ? 0 : step_exponent(amax);
    const float step = pow2f(-eq);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t pos[2], neg[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        pos[h] = neg[h] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t x = w[4 * i + 2 * h + j / 2];
          const float f = (j & 1 ? hi_bf16(x) : lo_bf16(x)) * step;
          const int v = none ? 0 : static_cast<int>(fminf(fmaxf(rintf(f), -127.f), 127.f));
          pos[h] |= (static_cast<uint32_t>(max(v, 0)) & 255u) << (8 * j);
          neg[h] |= (static_cast<uint32_t>(min(v, 0)) & 255u) << (8 * j);
        }
      }
      qb[i / 2][2 * (i % 2)] = static_cast<int>(pos[0]);
      qb[i / 2][2 * (i % 2) + 1] = static_cast<int>(pos[1]);
      qb[2 + i / 2][2 * (i % 2)] = static_cast<int>(neg[0]);
      qb[2 + i / 2][2 * (i % 2) + 1] = static_cast<int>(neg[1]);
    }
  }
  const int8_t* const sum = P.sum + static_cast<int64_t>(g) * P.nb * kSum;
  const int8_t* const exps = P.exp + static_cast<int64_t>(g) * P.nb;
  const int32_t* const table = P.tables + static_cast<int64_t>(b) * P.max_blocks;
  float* const to = P.scores + (static_cast<int64_t>(b) * P.H + g) * P.max_blocks;
#pragma unroll 1
  for (int i = 0; i < kTilesPerWave; ++i) {
    const int first = chunk * kScoreBlocks + (i * 4 + wave) * kTileBlocks;
    if (first >= n) break;  // uniform over the wavefront
    const int blk = first + r;
    int32_t id = blk < n ? table[blk] : -1;
    const bool ok = id >= 0 && id < P.nb;
    id = ok ? id : 0;
    i32x4 a[4] = {};
    if (ok) {
      const i32x4* s = reinterpret_cast<const i32x4*>(sum + static_cast<int64_t>(id) * kSum) + qd;
#pragma unroll
      for (int j = 0; j < 4; ++j) a[j] = s[4 * j];
    }
    const int e = ok ? exps[id] : -128;  // -128: no such block
    i32x4 c = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[j], qb[j], c, 0, 0, 0);
    // lane (column r, rows 4 qd ..): the row's exponent, the largest column
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int er = __shfl(e, 4 * qd + j, 64);
      float x = r < G ? ldexpf(static_cast<float>(c[j]), er + eq) : -INFINITY;
#pragma unroll
      for (int m = 8; m >= 1; m >>= 1) x = fmaxf(x, __shfl_xor(x, m, 64));
      v[j] = er == -128 ? -INFINITY : er == kNotFinite ? INFINITY : x;
    }
    if (r < 4 && first + 4 * qd + r < n)
      to[first + 4 * qd + r] = r == 0 ? v[0] : r == 1 ? v[1] : r == 2 ? v[2] : v[3];
  }
}

// The order of a score as an unsigned key; blocks that are always taken
// stand above every score.
__device__ __forceinline__ uint32_t key_of(const SelectParams& P, const float* scores, int i,
                                           int n) {
  if (i < P.n_first || i >= n - P.n_last) return 0xffffffffu;
  const uint32_t u = __float_as_uint(scores[i] + 0.f);  // -0 as 0: they are equal
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

// One workgroup per (request, KV head): the top_k-th largest key by its
// digits (256 bins, four passes), then the blocks above it and the first of
// those equal to it, in order.
constexpr int kSelThreads = 256;
__global__ __launch_bounds__(kSelThreads) void select_blocks_kernel(SelectParams P) {
  __shared__ int hist[256], s_wave[2][kSelThreads / 64], s_pick[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x / P.H;
  const int n = context_blocks(P, b);
  int32_t* const sel = P.sel + static_cast<int64_t>(blockIdx.x) * P.top_k;
  if (n <= P.top_k) {  // uniform: every block
    for (int i = tid; i < P.top_k; i += kSelThreads) sel[i] = i < n ? i : -1;
    return;
  }
  const float* const scores = P.scores + static_cast<int64_t>(blockIdx.x) * P.max_blocks;
  uint32_t prefix = 0;
  int need = P.top_k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kSelThreads) {
      const uint32_t k = key_of(P, scores, i, n);
      if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    // keys with a digit of at least 255 - tid
    const int own = hist[255 - tid];
    int x = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(x, d, 64);
      if (lane >= d) x += y;
    }
    if (lane == 63) s_wave[0][wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; ++w) x += s_wave[0][w];
    if (x >= need && x - own < need) {
      s_pick[0] = 255 - tid;
      s_pick[1] = need - (x - own);
    }
    __syncthreads();
    prefix |= static_cast<uint32_t>(s_pick[0]) << shift;
    need = s_pick[1];
    __syncthreads();
  }
  // need: how many of the keys equal to prefix are taken, lowest index first
  int above = 0, equal = 0;  // before this chunk
  for (int base = 0; base < n; base += kSelThreads) {
    const int i = base + tid;
    const uint32_t k = i < n ? key_of(P, scores, i, n) : 0;
    const bool gt = i < n && k > prefix, eq = i < n && k == prefix;
    const unsigned long long mg = __ballot(gt), me = __ballot(eq);
    if (lane == 0) {
      s_wave[0][wave] = __popcll(mg);
      s_wave[1][wave] = __popcll(me);
    }
    __syncthreads();
    int g0 = above, e0 = equal;
    for (int w = 0; w < kSelThreads / 64; ++w) {
      if (w < wave) {
        g0 += s_wave[0][w];
        e0 += s_wave[1][w];
      }
      above += s_wave[0][w];
      equal += s_wave[1][w];
    }
    const unsigned long long below = (1ull << lane) - 1;
    g0 += __popcll(mg & below);
    e0 += __popcll(me & below);
    if (gt || (eq && e0 < need)) sel[g0 + min(e0, need)] = i;
    __syncthreads();
  }
}

}  // namespace

using namespace bst;

extern "C" {

int boost_kv_index_enable(boost_kv_pool* p) {
  if (!p) return fail(BOOST_EINVAL, "null argument");
  if (p->ctx->device < 0 || !p->d_page_table) return fail(BOOST_ENODEV, "plan-only pool");
  if (p->cfg.head_dim != static_cast<uint32_t>(kD))
    return fail(BOOST_EINVAL, "block summaries need head_dim %d", kD);
  if (p->d_index) return BOOST_OK;
  BOOST_HIP(hipSetDevice(p->ctx->device));
  const uint64_t blocks = static_cast<uint64_t>(p->cfg.layers) * p->cfg.kv_heads * p->geom.nb;
  void* mem = nullptr;
  hipError_t e = hipMalloc(&mem, blocks * (kSum + 1));
  if (e == hipSuccess) e = hipMemset(mem, 0, blocks * (kSum + 1));
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    (void)hipFree(mem);
    return fail(e == hipErrorOutOfMemory ? BOOST_ENOMEM : BOOST_EHIP, "block summaries: %s",
                hipGetErrorString(e));
  }
  p->d_index = static_cast<int8_t*>(mem);
  return BOOST_OK;
}

int boost_kv_index_update(boost_ctx* ctx, const boost_kv_pool* p, int layer,
                          const int32_t* block_tables, int max_blocks, const int32_t* starts,
                          const int32_t* ends, int B, int max_tokens, void* stream) {
  if (!ctx || !p || !block_tables || !starts || !ends) return fail(BOOST_EINVAL, "null argument");
  const char* const *pk, * const *pv;
  if (int rc = kv_layer(p, layer, &pk, &pv)) return rc;
  if (!p->d_index) return fail(BOOST_EINVAL, "the pool has no block summaries");
  if (B < 1 || max_blocks < 1 || max_tokens < 1)
    return fail(BOOST_EINVAL, "B=%d max_blocks=%d max_tokens=%d", B, max_blocks, max_tokens);
  const int H = static_cast<int>(p->cfg.kv_heads);
  const uint64_t blocks = static_cast<uint64_t>(p->cfg.layers) * H * p->geom.nb;
  const uint64_t at = static_cast<uint64_t>(layer) * H * p->geom.nb;
  const IndexParams P{pk, p->d_index + at * kSum, p->d_index + blocks * kSum + at, block_tables,
                      starts, ends, B, H, static_cast<int>(p->geom.nb), max_blocks};
  // blocks that max_tokens new tokens can touch, one wavefront each (a
  // request with more has its wavefronts go round)
  const int64_t touched = std::min<int64_t>((static_cast<int64_t>(max_tokens) + 2 * kT - 2) / kT,
                                            max_blocks);
  const int chunks = static_cast<int>((touched + 3) / 4);
  const int64_t grid = static_cast<int64_t>(chunks) * B * H;
  if (grid > 0x7fffffff) return fail(BOOST_EINVAL, "grid too large");
  const auto kernel = p->format == BOOST_KV_FP4 ? index_update_kernel<true>
                                                : index_update_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(grid)), dim3(256), 0,
                     static_cast<hipStream_t>(stream), P, chunks);
  BOOST_HIP(hipGetLastError());
  return BOOST_OK;
}

int boost_kv_select(boost_ctx* ctx, const boost_kv_pool* p, int layer, const void* q, int B, int Hq,
                    const int32_t* block_tables, int max_blocks, const int32_t* ctx_lens,
                    int top_k, int n_first, int n_last, float* scores, int32_t* sel,
                    void* stream) {
  if (!ctx || !p || !q || !block_tables || !ctx_lens || !scores || !sel)
    return fail(BOOST_EINVAL, "null argument");
  const char* const *pk, * const *pv;
  if (int rc = kv_layer(p, layer, &pk, &pv)) return rc;
  if (!p->d_index) return fail(BOOST_EINVAL, "the pool has no block summaries");
  const int H = static_cast<int>(p->cfg.kv_heads);
  if (B < 1 || max_blocks < 1) return fail(BOOST_EINVAL, "B=%d max_blocks=%d", B, max_blocks);
  if (Hq < H || Hq % H || Hq / H > 16)
    return fail(BOOST_EINVAL, "Hq=%d: a multiple of %d KV heads, up to 16 of each", Hq, H);
  if (top_k < 1 || n_first < 0 || n_last < 0 ||
      static_cast<int64_t>(n_first) + n_last > top_k)
    return fail(BOOST_EINVAL, "top_k=%d n_first=%d n_last=%d", top_k, n_first, n_last);
  if (reinterpret_cast<uintptr_t>(q) & 15) return fail(BOOST_EINVAL, "q must be 16-byte aligned");
  const uint64_t blocks = static_cast<uint64_t>(p->cfg.layers) * H * p->geom.nb;
  const uint64_t at = static_cast<uint64_t>(layer) * H * p->geom.nb;
  const SelectParams P{p->d_index + at * kSum, p->d_index + blocks * kSum + at,
                       static_cast<const uint16_t*>(q), block_tables, ctx_lens, scores, sel, B, H,
                       Hq, static_cast<int>(p->geom.nb), max_blocks, top_k, n_first, n_last};
  const int chunks = (max_blocks + kScoreBlocks - 1) / kScoreBlocks;
  const int64_t grid = static_cast<int64_t>(chunks) * B * H;
  if (grid > 0x7fffffff) return fail(BOOST_EINVAL, "grid too large");
  const auto s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(block_scores_kernel, dim3(static_cast<unsigned>(grid)), dim3(256), 0, s, P,
                     chunks);
  BOOST_HIP(hipGetLastError());
  hipLaunchKernelGGL(select_blocks_kernel, dim3(static_cast<unsigned>(B) * H), dim3(kSelThreads),
                     0, s, P);
  BOOST_HIP(hipGetLastError());
  return BOOST_OK;
}

}  // extern "C"
