// Block summaries of a KV pool and the selection of blocks by them: what
// sparse attention reads in place of a long context.
//
// Summary of a head-block: for every dim the largest and the smallest key of
// its live tokens, outwards in whole steps of 2^e, e the smallest (>= -126)
// with max|k| <= 127 * 2^e:
//   hi_d = ceil(max_t k_td / 2^e)   lo_d = floor(min_t k_td / 2^e)
// kept as int8 hi_d and -lo_d, so that both meet magnitudes of q8 below.
// Score of a block for a query head: q8 = round(q / 2^eq) (the same rule for
// eq, ties to even, at most 127), 2^(e + eq) sum_d max(q8_d hi_d, q8_d lo_d),
// an upper bound of q8 . k over the block's tokens; for a KV head the largest
// over its query heads.  The sum is one of whole numbers below 2^21 and the
// factor a power of two, so a score is exact and a selection does not depend
// on the order of any sum: the same blocks on every placement, split and
// machine.  257 bytes stand for the 8 KiB (bf16) of a head-block.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kvfmt.h"
#include "runtime.h"

namespace {

constexpr int kD = 128;
constexpr int kT = 16;
constexpr int kSum = 2 * kD;      // bytes of a summary: hi, then -lo
constexpr int kNotFinite = 127;   // exponent byte of a block with an inf or NaN key

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

struct IndexParams {
  bst::KPages pages;        // this layer's
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

// Two bf16 values as two 16-bit integers in the same order (its own inverse;
// NaNs lie beyond the infinities of their sign), so that two extremes take one
// instruction each.
typedef __attribute__((ext_vector_type(2))) short i16x2;
__device__ __forceinline__ i16x2 ordered(uint32_t v) {
  const i16x2 x = __builtin_bit_cast(i16x2, v);
  return x ^ ((x >> 15) & static_cast<short>(0x7fff));
}
__device__ __forceinline__ uint32_t values_of(i16x2 x) {
  return __builtin_bit_cast(uint32_t, x ^ ((x >> 15) & static_cast<short>(0x7fff)));
}
__device__ __forceinline__ i16x2 max2(i16x2 a, i16x2 b) { return __builtin_elementwise_max(a, b); }
__device__ __forceinline__ i16x2 min2(i16x2 a, i16x2 b) { return __builtin_elementwise_min(a, b); }
constexpr short kNone = -32768;  // below every value (and, negated less one, above)

// The value of another lane of the 16-lane row: CTRL is a DPP pattern.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return static_cast<uint32_t>(
      __builtin_amdgcn_mov_dpp(static_cast<int>(v), CTRL, 0xf, 0xf, true));
}
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kXor7 = 0x141, kXor8 = 0x128;
template <int CTRL>
__device__ __forceinline__ i16x2 dpp2(i16x2 v) {
  return __builtin_bit_cast(i16x2, dpp<CTRL>(__builtin_bit_cast(uint32_t, v)));
}
// The largest v of the row's 16 lanes, in each of them.
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  v = max(v, dpp<kXor1>(v));
  v = max(v, dpp<kXor2>(v));
  v = max(v, dpp<kXor7>(v));
  return max(v, dpp<kXor8>(v));
}
// v of the lanes 16 and 32 apart by f.
template <typename F>
__device__ __forceinline__ uint32_t over_rows(uint32_t v, F f) {
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = f(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return f(b[0], b[1]);
}

template <typename F>
__device__ __forceinline__ i16x2 over_rows2(i16x2 v, F f) {
  return __builtin_bit_cast(i16x2, over_rows(__builtin_bit_cast(uint32_t, v), [&](uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, f(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
  }));
}

// v in whole steps of 1 / scale, rounded up: one step at least for a positive v
// (the product is 0 where it is below every fp32 number).
__device__ __forceinline__ int steps_up(float v, float scale) {
  const int n = static_cast<int>(ceilf(v * scale));
  return v > 0.f ? max(n, 1) : n;
}

// The larger magnitude, as bf16 bits, of extremes hi (largest) and lo
// (smallest) in both halves.
__device__ __forceinline__ uint32_t magnitude(i16x2 hi, i16x2 lo) {
  const uint32_t h = values_of(hi), l = values_of(lo);
  // the magnitude of the largest value counts if it is not negative, that of
  // the smallest if it is
  auto one = [](uint32_t hv, uint32_t lv) {
    const uint32_t a = hv & 0x8000u ? 0u : hv, b = lv & 0x8000u ? lv & 0x7fffu : 0u;
    return max(a, b);
  };
  return max(one(h & 0xffffu, l & 0xffffu), one(h >> 16, l >> 16));
}

__device__ __forceinline__ const char* page_at(const bst::KPages& L, uint32_t page) {
  const bool host = page >= L.first_host;
  return (host ? L.host : L.hbm) + (static_cast<uint64_t>(host ? page - L.first_host : page) << 21);
}

// One wavefront per head-block.  FP4: lane (token r, group qd); else lane
// (8-dim chunk r, token row qd of four).  Bound by the keys' bytes: the
// extremes of two dims take one instruction, and no lane's value goes through
// LDS.  104 MB of keys (four prompts of 9001..16384 tokens, 8 heads, bf16): 21
// us, 4.7 TB/s (33 through LDS; two blocks a wavefront at a time 2 us more); the
// last blocks of 16 requests 3.6.
template <bool FP4>
__global__ __launch_bounds__(256) void index_update_kernel(IndexParams P) {
  const int lane = threadIdx.x & 63, r = lane & 15, qd = lane >> 4;
  const int b = blockIdx.z, g = blockIdx.y, chunk = blockIdx.x, chunks = gridDim.x;
  const int start = max(P.starts[b], 0);
  const int end = static_cast<int>(
      min(static_cast<int64_t>(P.ends[b]), static_cast<int64_t>(P.max_blocks) * kT));
  if (start >= end) return;
  const int last = (end - 1) / kT;
  for (int blk = start / kT + chunk * 4 + static_cast<int>(threadIdx.x >> 6); blk <= last;
       blk += chunks * 4) {
    const int32_t id = __builtin_amdgcn_readfirstlane(
        P.tables[static_cast<int64_t>(b) * P.max_blocks + blk]);
    if (id < 0 || id >= P.nb) continue;  // uniform over the wavefront
    const int live = min(kT, end - blk * kT);
    const int64_t at = static_cast<int64_t>(g) * P.nb + id;
    int8_t* const out = P.sum + at * kSum;
    if constexpr (FP4) {
      using namespace bst;
      const Fp4At f = fp4_at(g, id, P.nb);
      const char* const page = page_at(P.pages, f.page);
      const uint4 c = *reinterpret_cast<const uint4*>(page + f.idx * kFp4Code + lane * 16);
      const float s = fp4_scale(
          static_cast<uint8_t>(page[kFp4ScaleAt + f.idx * kFp4Scale + lane]));
      const bool in = r < live;
      const uint32_t w[4] = {c.x, c.y, c.z, c.w};
      i16x2 mx[16], mn[16];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t v[4] = {fp4_unpack<0>(w[i], s), fp4_unpack<1>(w[i], s),
                               fp4_unpack<2>(w[i], s), fp4_unpack<3>(w[i], s)};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const i16x2 x = ordered(v[j]);
          mx[4 * i + j] = in ? x : i16x2{kNone, kNone};
          mn[4 * i + j] = in ? x : i16x2{-1 - kNone, -1 - kNone};
        }
      }
      // over the 16 tokens, half of the dims kept in each step: lane r ends
      // with dims 2 r, 2 r + 1 of its group
      auto step = [&](auto ctrl, auto count, bool up) {
        constexpr int C = decltype(ctrl)::value, N = decltype(count)::value;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const i16x2 kx = up ? mx[N + i] : mx[i], gx = up ? mx[i] : mx[N + i];
          const i16x2 kn = up ? mn[N + i] : mn[i], gn = up ? mn[i] : mn[N + i];
          mx[i] = max2(kx, dpp2<C>(gx));
          mn[i] = min2(kn, dpp2<C>(gn));
        }
      };
      using std::integral_constant;
      // (lanes xor 8, 7, 2, 1: together all 16 of a row)
      step(integral_constant<int, kXor8>{}, integral_constant<int, 8>{}, lane & 8);
      step(integral_constant<int, kXor7>{}, integral_constant<int, 4>{}, lane & 4);
      step(integral_constant<int, kXor2>{}, integral_constant<int, 2>{}, lane & 2);
      step(integral_constant<int, kXor1>{}, integral_constant<int, 1>{}, lane & 1);
      uint32_t amax = row_max(magnitude(mx[0], mn[0]));
      amax = over_rows(amax, [](uint32_t a, uint32_t b) { return max(a, b); });
      const bool bad = amax >= 0x7f80;  // no numbers to keep
      const int e = bad ? kNotFinite : step_exponent(amax);
      const float scale = pow2f(bad ? 0 : -e);
      const uint32_t hx = values_of(mx[0]), hn = values_of(mn[0]);
      const char2 hi = {static_cast<signed char>(steps_up(lo_bf16(hx), scale)),
                        static_cast<signed char>(steps_up(hi_bf16(hx), scale))};
      const char2 lo = {static_cast<signed char>(steps_up(-lo_bf16(hn), scale)),
                        static_cast<signed char>(steps_up(-hi_bf16(hn), scale))};
      int8_t* const o = out + 32 * qd + 2 * r;
      *reinterpret_cast<char2*>(o) = bad ? char2{0, 0} : hi;
      *reinterpret_cast<char2*>(o + kD) = bad ? char2{0, 0} : lo;
      if (lane == 0) P.exp[at] = static_cast<int8_t>(e);
    } else {
      const uint64_t byte = static_cast<uint64_t>(at) * kT * kD * 2;
      const char* const src = page_at(P.pages, static_cast<uint32_t>(byte >> 21)) +
                              (byte & (bst::kPage - 1)) + lane * 16;
      u32x4 u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)  // token 4 i + qd
        u[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + i * 1024));
      i16x2 mx[4], mn[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        mx[j] = i16x2{kNone, kNone};
        mn[j] = i16x2{-1 - kNone, -1 - kNone};
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool in = 4 * i + qd < live;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const i16x2 x = ordered(u[i][j]);
          mx[j] = max2(mx[j], in ? x : i16x2{kNone, kNone});
          mn[j] = min2(mn[j], in ? x : i16x2{-1 - kNone, -1 - kNone});
        }
      }
      uint32_t amax = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        mx[j] = over_rows2(mx[j], max2);
        mn[j] = over_rows2(mn[j], min2);
        amax = max(amax, magnitude(mx[j], mn[j]));
      }
      amax = row_max(amax);
      const bool bad = amax >= 0x7f80;
      const int e = bad ? kNotFinite : step_exponent(amax);
      const float scale = pow2f(bad ? 0 : -e);
      uint32_t w[2] = {0, 0};
      if (!bad) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t v = values_of(qd == 0 ? mx[j] : mn[j]);
          const int p = steps_up(qd == 0 ? lo_bf16(v) : -lo_bf16(v), scale);
          const int q = steps_up(qd == 0 ? hi_bf16(v) : -hi_bf16(v), scale);
          w[j / 2] |= ((static_cast<uint32_t>(p) & 255u) | (static_cast<uint32_t>(q) & 255u) << 8)
                      << (16 * (j % 2));
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

// Scores of 16-block tiles, four to a wavefront: rows are the KV head's query
// heads, columns blocks, the 256 products of a pair in four 16x16x64 integer
// products (hi against the positive part of q8, -lo against the magnitude of
// the negative one), so that a lane ends with four heads of one block.  Bound by
// the summaries' bytes and the chain before them (block ids): the loads of all
// four tiles are out together, and q is rounded while they are, a quarter by
// each wavefront.  33 MB (16 requests of 2000..30000 tokens, 8 heads) 11.8 us,
// one of 131072 tokens 4.8.
constexpr int kTileBlocks = 16, kTiles = 4;
constexpr int kScoreBlocks = 4 * kTileBlocks * kTiles;  // per workgroup

// A workgroup's (4 or 8 wavefronts') share of the scores of (request b, KV head
// g): blocks from `base` on, to P.scores and, if not null, s_score[block].
// Returns the context's blocks.
__device__ __forceinline__ int scores_from(const SelectParams& P, int b, int g, int base,
                                           float* s_score) {
  // the operand of q by lane: dword w of 16 dims of step s (positive parts of
  // the lower and the upper 64 dims, then the negative ones)
  __shared__ uint32_t s_q[4][64][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, qd = lane >> 4;
  const int quarter = wave & 3;  // of the rounding of q (of eight wavefronts two write the same of it)
  const int L = P.lens[b];  // (the ids do not wait for it)
  const int first = base + wave * kTiles * kTileBlocks;
  const int G = P.Hq / P.H;
  const int8_t* const sum = P.sum + static_cast<int64_t>(g) * P.nb * kSum;
  const int8_t* const exps = P.exp + static_cast<int64_t>(g) * P.nb;
  const int32_t* const table = P.tables + static_cast<int64_t>(b) * P.max_blocks;
  int32_t id[kTiles];
  i32x4 a[kTiles][4];
  int e[kTiles];  // of block (column) r; -128: no such block
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
    id[i] = table[min(first + i * kTileBlocks + r, P.max_blocks - 1)];
  // row r: head r (beyond G the last again), dims 16 qd .. + 15 and 64 more
  uint32_t w[16];
  {
    const uint4* q = reinterpret_cast<const uint4*>(
        P.q + (static_cast<int64_t>(b) * P.Hq + g * G + min(r, G - 1)) * kD + 16 * qd);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 u = q[i < 2 ? i : 6 + i];  // 64 dims are 8 uint4 further
      w[4 * i] = u.x;
      w[4 * i + 1] = u.y;
      w[4 * i + 2] = u.z;
      w[4 * i + 3] = u.w;
    }
  }
  const int n = L <= 0 ? 0 : min((L - 1) / kT + 1, P.max_blocks);
  if (base >= n) return n;  // uniform
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    const bool ok = first + i * kTileBlocks + r < n && id[i] >= 0 && id[i] < P.nb;
    id[i] = ok ? id[i] : 0;
    const i32x4* s = reinterpret_cast<const i32x4*>(sum + static_cast<int64_t>(id[i]) * kSum) + qd;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[i][j] = s[4 * j];
    e[i] = exps[id[i]];
    e[i] = ok ? e[i] : -128;
  }
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) amax = max(amax, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
  amax = over_rows(amax, [](uint32_t x, uint32_t y) { return max(x, y); });
  const bool none = amax >= 0x7f80;  // a query that is not finite counts as 0
  const int eq = none ? 0 : step_exponent(amax);
  const float step = pow2f(-eq);
#pragma unroll
  for (int h = 0; h < 2; ++h) {  // this wavefront's four dims of the lower and upper 64
    uint32_t x0 = w[8 * h], x1 = w[8 * h + 1];
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      x0 = quarter == i ? w[8 * h + 2 * i] : x0;
      x1 = quarter == i ? w[8 * h + 2 * i + 1] : x1;
    }
    // whole numbers up to 127 by the rule of eq; the conversion has 0 for
    // what is below 0
    const float f[4] = {rintf(lo_bf16(x0) * step), rintf(hi_bf16(x0) * step),
                        rintf(lo_bf16(x1) * step), rintf(hi_bf16(x1) * step)};
    uint32_t pos = 0, neg = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      pos = __builtin_amdgcn_cvt_pk_u8_f32(f[j], j, pos);
      neg = __builtin_amdgcn_cvt_pk_u8_f32(-f[j], j, neg);
    }
    s_q[h][lane][quarter] = none ? 0 : pos;
    s_q[2 + h][lane][quarter] = none ? 0 : neg;
  }
  __syncthreads();
  if (first >= n) return n;  // uniform over the wavefront; no barrier follows
  i32x4 qb[4];
  int eq4[4];  // of heads (rows) 4 qd ..
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    qb[s] = *reinterpret_cast<const i32x4*>(s_q[s][lane]);
    eq4[s] = __shfl(eq, 4 * qd + s, 64);
  }
  float* const to = P.scores + (static_cast<int64_t>(b) * P.H + g) * P.max_blocks;
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    const int row0 = first + i * kTileBlocks;
    if (row0 >= n) break;  // uniform over the wavefront
    i32x4 c = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_i32_16x16x64_i8(qb[j], a[i][j], c, 0, 0, 0);
    float v = -INFINITY;  // the largest of up to 16 heads
#pragma unroll
    for (int j = 0; j < 4; ++j) v = fmaxf(v, ldexpf(static_cast<float>(c[j]), e[i] + eq4[j]));
    if (G > 4)  // uniform: rows past the fourth are other heads
      v = __uint_as_float(over_rows(__float_as_uint(v), [](uint32_t x, uint32_t y) {
        return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y)));
      }));
    v = e[i] == -128 ? -INFINITY : e[i] == kNotFinite ? INFINITY : v;
    if (qd == 0 && row0 + r < n) {
      to[row0 + r] = v;
      if (s_score) s_score[row0 + r] = v;
    }
  }
  return n;
}

__global__ __launch_bounds__(256) void block_scores_kernel(SelectParams P) {
  scores_from(P, blockIdx.z, blockIdx.y, blockIdx.x * kScoreBlocks, nullptr);
}

// Sum of v over this lane and those before it.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // the lane before, in its row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);  // 2 before
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);  // 4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);  // 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row 0 to 1, 2 to 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // rows 0 and 1 to 2 and 3
  return v;
}

// One workgroup per (request, KV head): the top_k-th largest key by its
// digits, then the keys above it and the first of those equal to it, in order.
// Thread t holds keys t, NT + t, ..., V of them in registers (those past
// V * NT blocks are read again in every pass).  The digits start at the
// highest bit in which any two keys differ (scores of one query differ little
// in their exponents: from bit 31 on, most keys would meet in one counter) and
// end when no key is left to decide.  Bound by the instructions of its few
// wavefronts between its barriers, not by the 4 bytes a block: nothing
// branches on a key, a digit is one barrier (every wavefront sums the counters
// for itself) and has counters of its own, four of each so that equal digits
// do not all wait for one another.  8 lists of 128 among 8192 blocks 6.9 us
// (12.5 with two barriers and branches), 128 of 64 among up to 1875 5.1.
// score(i): that of block i of n; list: its number among [B, H].
template <int NT, int V, typename Score>
__device__ __forceinline__ void select_list(const SelectParams& P, int64_t list, int n, Score score) {
  constexpr int kWaves = NT / 64, kRound = 64;  // chunks of NT keys ranked at a time
  constexpr int kCopies = 4, kDigits = 4, kCounters = 256 * kCopies;
  // of each digit, and 64 that nothing reads, for keys that do not count
  __shared__ __align__(16) int hist[kDigits * kCounters + 64];
  __shared__ int s_cnt[kRound * (kWaves + 1)];  // above | equal << 16, of a chunk's wavefronts
  __shared__ uint32_t s_bits[2][kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t* const sel = P.sel + list * P.top_k;
  if (n <= P.top_k) {  // uniform: every block
    for (int i = tid; i < P.top_k; i += NT) sel[i] = i < n ? i : -1;
    return;
  }
  // the key of blocks that are always taken; no score's (it would be a NaN's)
  constexpr uint32_t kAlways = 0xffffffffu;
  auto key_of = [&](float v, int i) {
    const uint32_t u = __float_as_uint(v + 0.f);  // -0 as 0: they are equal
    const uint32_t k = u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
    return i < P.n_first || i >= n - P.n_last ? kAlways : k;
  };
  auto key_at = [&](int i) { return key_of(score(i), i); };
  const int chunks = (n + NT - 1) / NT;
  uint32_t key[V];
  float own[V];  // loaded without a branch, all of them together
#pragma unroll
  for (int j = 0; j < V; ++j) own[j] = score(min(j * NT + tid, n - 1));
  for (int i = tid; i < kDigits * kCounters / 4; i += NT)
    reinterpret_cast<i32x4*>(hist)[i] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const uint32_t k = key_of(own[j], j * NT + tid);
    key[j] = j * NT + tid < n ? k : kAlways;
  }
  auto each = [&](auto f) {  // kAlways among them
#pragma unroll
    for (int j = 0; j < V; ++j) f(key[j]);
    for (int i = V * NT + tid; i < n; i += NT) f(key_at(i));
  };
  // bits in which keys differ: set in one and clear in another
  uint32_t any1 = 0, any0 = 0;
  each([&](uint32_t k) {
    any1 |= k == kAlways ? 0u : k;
    any0 |= ~k;  // (of kAlways: none)
  });
  auto either = [](uint32_t x, uint32_t y) { return x | y; };
  auto over_wave = [&](uint32_t v) {
    v |= dpp<kXor1>(v);
    v |= dpp<kXor2>(v);
    v |= dpp<kXor7>(v);
    v |= dpp<kXor8>(v);
    return over_rows(v, either);
  };
  any1 = over_wave(any1);
  any0 = over_wave(any0);
  if (lane == 0) {
    s_bits[0][wave] = any1;
    s_bits[1][wave] = any0;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    any1 |= s_bits[0][w];
    any0 |= s_bits[1][w];
  }
  const uint32_t differ = any1 & any0;
  int top = differ ? 32 - __clz(static_cast<int>(differ)) : 0;  // undecided bits
  // the decided bits of the last key that is taken; at first those all share
  uint32_t least = top == 32 ? 0 : (any1 & ~any0) >> top << top;
  // how many are taken of the keys with these bits (n > top_k: the first and
  // the last blocks are apart)
  int need = P.top_k - P.n_first - P.n_last;
  bool open = need > 0;
  for (int* h = hist; open && top > 0; h += kCounters) {  // at most four digits
    const int shift = max(0, top - 8);
    const uint32_t digit = (1u << (top - shift)) - 1, decided = top == 32 ? 0u : ~0u << top;
    const uint32_t mine = lane % kCopies;
    const uint32_t out = static_cast<uint32_t>(hist + kDigits * kCounters - h) + lane;
    each([&](uint32_t k) {
      const uint32_t d = (k >> shift & digit) * kCopies + mine;
      atomicAdd(&h[((k ^ least) & decided) == 0 && k != kAlways ? d : out], 1);
    });
    __syncthreads();
    // lane l: digits 255 - 4 l, ... - 3, with the keys above them
    int c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const i32x4 u = *reinterpret_cast<const i32x4*>(&h[(255 - 4 * lane - j) * kCopies]);
      c[j] = u[0] + u[1] + u[2] + u[3];
    }
    const int x = c[0] + c[1] + c[2] + c[3], upto = wave_scan(x);
    int before = upto - x, pick = 0, take = 0, count = 0;
    const int l = __ffsll(__ballot(before < need && upto >= need)) - 1;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool here = before < need && before + c[j] >= need;
      pick = here ? 255 - 4 * lane - j : pick;
      take = here ? need - before : take;
      count = here ? c[j] : count;
      before += c[j];
    }
    least |= static_cast<uint32_t>(__builtin_amdgcn_readlane(pick, l)) << shift;
    need = __builtin_amdgcn_readlane(take, l);
    open = __builtin_amdgcn_readlane(count, l) != need;  // else every key of this digit is taken
    top = shift;
  }
  // keys above `upto` are taken, and the first `need` from least to there
  const uint32_t upto = P.top_k == P.n_first + P.n_last ? kAlways - 1
                        : least | (top >= 32 ? 0xffffffffu : (1u << top) - 1);
  if (P.top_k == P.n_first + P.n_last) least = kAlways;
  int above0 = 0, equal0 = 0;  // before this round
  for (int c0 = 0; c0 < chunks; c0 += kRound) {
    const int m = min(kRound, chunks - c0);
    // lane j: this wavefront's 64 blocks of chunk j that are above, and equal
    unsigned long long gt_own = 0, eq_own = 0;
    auto mark = [&](int j, uint32_t k, bool in) {  // all lanes together
      const bool more = in && (k > upto || k == kAlways);
      const unsigned long long x = __ballot(more), y = __ballot(in && !more && k >= least);
      gt_own = lane == j ? x : gt_own;
      eq_own = lane == j ? y : eq_own;
    };
    if (c0 == 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) mark(j, key[j], j * NT + tid < n);
    }
    for (int j = c0 == 0 ? V : 0; j < m; ++j) {
      const int i = (c0 + j) * NT + tid;
      mark(j, key_at(min(i, n - 1)), i < n);
    }
    if (c0 > 0) __syncthreads();  // s_cnt is free again
    s_cnt[lane * (kWaves + 1) + wave] = __popcll(gt_own) | __popcll(eq_own) << 16;
    __syncthreads();
    // what stands before: in the chunk, then in the chunks before it
    int x = 0, y = 0, own_x = 0, own_y = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int c = s_cnt[lane * (kWaves + 1) + w];
      own_x = w == wave ? x : own_x;
      own_y = w == wave ? y : own_y;
      x += c & 0xffff;
      y += c >> 16;
    }
    const int sx = wave_scan(x), sy = wave_scan(y);
    own_x += above0 + sx - x;
    own_y += equal0 + sy - y;
    above0 += __builtin_amdgcn_readlane(sx, 63);
    equal0 += __builtin_amdgcn_readlane(sy, 63);
    // the words again by all lanes: of a round of up to 4, 16 or 64 chunks a
    // lane has so many bits of one word, and writes those that are taken
    const int lg = m <= 4 ? 2 : m <= 16 ? 4 : 6;
    const int j = lane >> (6 - lg), from = (lane & ((64 >> lg) - 1)) << lg;
    unsigned long long gt = __shfl(gt_own, j, 64), eq = __shfl(eq_own, j, 64);
    const unsigned long long below = (1ull << from) - 1, bits = ~0ull >> (64 - (1 << lg));
    int a = __shfl(own_x, j, 64) + static_cast<int>(__popcll(gt & below));
    int e = __shfl(own_y, j, 64) + static_cast<int>(__popcll(eq & below));
    gt = gt >> from & bits;
    eq = e < need ? eq >> from & bits : 0;
    const int i0 = (c0 + j) * NT + 64 * wave + from;
    for (unsigned long long left = gt | eq; left; left &= left - 1) {
      const int i = __ffsll(left) - 1;
      const bool above = gt >> i & 1;
      if (above || e < need) sel[a + min(e, need)] = i0 + i;
      a += above;
      e += !above;
    }
  }
}

template <int NT, int V>
__global__ __launch_bounds__(NT) void select_blocks_kernel(SelectParams P) {
  const float* const scores = P.scores + static_cast<int64_t>(blockIdx.x) * P.max_blocks;
  select_list<NT, V>(P, blockIdx.x, context_blocks(P, blockIdx.x / P.H),
                     [&](int i) { return scores[i]; });
}

// Both in one launch, for tables whose scores one workgroup of W wavefronts
// computes in a round.
template <int W>
__global__ __launch_bounds__(64 * W) void scores_select_kernel(SelectParams P) {
  constexpr int kBlocks = W * kTiles * kTileBlocks;
  __shared__ float s_score[kBlocks];
  const int g = blockIdx.x, b = blockIdx.y;
  const int n = scores_from(P, b, g, 0, s_score);
  __syncthreads();
  select_list<64 * W, kBlocks / (64 * W)>(P, static_cast<int64_t>(b) * P.H + g, n,
                                          [&](int i) { return s_score[i]; });
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
  KPages pages;
  if (int rc = k_pages(p, layer, pages)) return rc;
  if (!p->d_index) return fail(BOOST_EINVAL, "the pool has no block summaries");
  if (B < 1 || max_blocks < 1 || max_tokens < 1)
    return fail(BOOST_EINVAL, "B=%d max_blocks=%d max_tokens=%d", B, max_blocks, max_tokens);
  const int H = static_cast<int>(p->cfg.kv_heads);
  const uint64_t blocks = static_cast<uint64_t>(p->cfg.layers) * H * p->geom.nb;
  const uint64_t at = static_cast<uint64_t>(layer) * H * p->geom.nb;
  const IndexParams P{pages, p->d_index + at * kSum, p->d_index + blocks * kSum + at, block_tables,
                      starts, ends, B, H, static_cast<int>(p->geom.nb), max_blocks};
  // blocks that max_tokens new tokens can touch, one wavefront each (a
  // request with more has its wavefronts go round; 2^22 of them are as many as
  // any card has work for, and a grid counts its threads in 32 bits)
  const int64_t touched = std::min<int64_t>({(static_cast<int64_t>(max_tokens) + 2 * kT - 2) / kT,
                                             max_blocks, 1 << 22});
  const int chunks = static_cast<int>((touched + 3) / 4);
  if (H > 65535 || B > 65535) return fail(BOOST_EINVAL, "grid too large");
  const auto kernel = p->format == BOOST_KV_FP4 ? index_update_kernel<true>
                                                : index_update_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3(chunks, H, B), dim3(256), 0, static_cast<hipStream_t>(stream), P);
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
  if (top_k < 1 || top_k > kMaxTop || n_first < 0 || n_last < 0 ||
      static_cast<int64_t>(n_first) + n_last > top_k)
    return fail(BOOST_EINVAL, "top_k=%d n_first=%d n_last=%d", top_k, n_first, n_last);
  if (reinterpret_cast<uintptr_t>(q) & 15) return fail(BOOST_EINVAL, "q must be 16-byte aligned");
  const uint64_t blocks = static_cast<uint64_t>(p->cfg.layers) * H * p->geom.nb;
  const uint64_t at = static_cast<uint64_t>(layer) * H * p->geom.nb;
  const SelectParams P{p->d_index + at * kSum, p->d_index + blocks * kSum + at,
                       static_cast<const uint16_t*>(q), block_tables, ctx_lens, scores, sel, B, H,
                       Hq, static_cast<int>(p->geom.nb), max_blocks, top_k, n_first, n_last};
  // a context has at most kMaxTop blocks, however wide the table is (block
  // numbers stay far below 2^31)
  const int chunks = (std::min(max_blocks, kMaxTop) + kScoreBlocks - 1) / kScoreBlocks;
  if (H > 65535 || B > 65535 || static_cast<int64_t>(B) * H > 0x7fffffff)
    return fail(BOOST_EINVAL, "grid too large");
  const auto s = static_cast<hipStream_t>(stream);
  // Tables of up to 512 blocks in one launch (whole steps: one request of 250
  // blocks 17.9 us, 19.5 with two launches; 64 of 250 43.6 and 45.6; 24 of 500
  // in 4 bits 20.5 and 22.1).  Few lists of the widest of these tables lose a
  // little (four of 500 18.9 and 18.2), which is accepted for a rule on the
  // width alone.  1000 blocks to a workgroup: one request 25.9 and 20.4.
  if (max_blocks <= 512) {
    if (max_blocks <= 256)
      hipLaunchKernelGGL(scores_select_kernel<4>, dim3(H, B), dim3(256), 0, s, P);
    else
      hipLaunchKernelGGL(scores_select_kernel<8>, dim3(H, B), dim3(512), 0, s, P);
    BOOST_HIP(hipGetLastError());
    return BOOST_OK;
  }
  hipLaunchKernelGGL(block_scores_kernel, dim3(chunks, H, B), dim3(256), 0, s, P);
  BOOST_HIP(hipGetLastError());
  // keys in registers as far as they go, and no more wavefronts than have work
  // (whole steps: 16 requests of up to 1875 blocks 44.8 us with 512 threads, 46.2
  // with 1024; one of 8192 28.1 with 512, 28.8 with 1024 and 30.6 with 256; one
  // of 31250 45.5 with 32 keys a thread, 54.5 with 16 and the rest read again in
  // every pass)
  const dim3 rows(static_cast<unsigned>(B) * H);
  if (max_blocks <= 2048)
    hipLaunchKernelGGL((select_blocks_kernel<512, 4>), rows, dim3(512), 0, s, P);
  else if (max_blocks <= 8192)
    hipLaunchKernelGGL((select_blocks_kernel<512, 16>), rows, dim3(512), 0, s, P);
  else
    hipLaunchKernelGGL((select_blocks_kernel<1024, 32>), rows, dim3(1024), 0, s, P);
  BOOST_HIP(hipGetLastError());
  return BOOST_OK;
}

}  // extern "C"
