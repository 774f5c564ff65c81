// a5 over a 4-bit pool: GQA paged-attention decode whose K and V are E2M1
// codes with a power-of-two scale per token and 32 dims (kvfmt.h).
//
// Work items, partitions and the merge are those of the bf16 kernel
// (attn_items.h).  Within an item every wavefront takes pairs of blocks (32
// tokens) in turn, on the matrix cores:
//
//   scores  S[t, c] = sum_d K[t, d] q[c, d], one 16x16x32 product per group of
//           8 dims of each quad: lane (r, qd) holds token r's codes of group
//           qd, one 16-byte load, converted to bf16 with the group's scale
//           (exact: a code has two significant bits, the scale is a power of
//           two).  q is bf16, so every product is exact and the sum is fp32.
//   softmax the result leaves tokens 4 qd .. 4 qd + 3 of column c in a lane;
//           running maximum and sum per column in fp32.
//   output  O[d, c] += sum_t V[t, d] p[t, c]: the probabilities stay in the
//           lanes that computed them, because the sum over t may run in any
//           order as long as V's operand follows it: lane (r, qd) holds tokens
//           4 qd .. 4 qd + 3 of dims 16 i + r (i = 0..7), again one 16-byte load.
//
// Columns: a call has G = Hq / H query heads to 16 columns, so head j also
// stands in columns G + j and 2 G + j, and each copy multiplies V by another
// part of the fp32 probability (its first 8 significant bits, the next 8, the
// rest; with G > 5 there are two copies and the second holds the rest rounded
// to 8 bits).  The parts' outputs are added in fp32 at the end: the precision
// of fp32 probabilities (G > 5: 16 to 17 bits) at no further matrix work.
#include <cmath>

#include "attn_items.h"
#include "kvfmt.h"

namespace {

using namespace bst::attn;
using bst::fp4_unpack;

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kCols = 16;
constexpr int kAccRow = kD + 4;  // floats of a column's row in LDS (banks)

__device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Maximum (or sum) of v over the four lanes that hold one column.
__device__ __forceinline__ float col_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float col_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// One block's codes and scales in a lane.
struct Block4 {
  u32x4 k, v;   // 32 codes of token r, group qd; four tokens of dims 16 i + r
  u32x4 vs;     // scale bytes of tokens 4 qd .. 4 qd + 3, a byte per group
  uint32_t ks;  // scale byte of token r, group qd
  int tok;      // tokens that count (0: none, nothing was read)
};

template <int PARTS, bool WAVE, bool SEL>
__global__ __launch_bounds__(kThreads) void attn4_partition(AttnParams P) {
  __shared__ float s_acc[4][kCols][kAccRow];
  __shared__ float s_ml[4][kCols][2];
  __shared__ int32_t row[kMaxPartBlocks];    // the partition's pool blocks
  __shared__ int32_t s_tok[kMaxPartBlocks];  // and their tokens that count
  __shared__ int s_red[4], s_pick[5];
  int part, b, g, L;
  if constexpr (WAVE) {
    if (!item_of_wave(P, blockIdx.x, b, g, part, L)) return;  // uniform
  } else {
    if (!item_of(P, blockIdx.x, b, g, part, L, s_red, row, s_pick)) return;  // uniform
  }
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r = lane & 15, qd = lane >> 4;
  const int G = P.Hq / P.H;
  const int n_blk = L <= 0 ? 0 : min((L + kT - 1) / kT, P.item_blocks);
  const int blk_beg = part * P.part_blocks;
  if (blk_beg >= n_blk) return;  // uniform
  const int nbp = min(n_blk, blk_beg + P.part_blocks) - blk_beg;
  __syncthreads();  // row has served the item search
  if (tid < nbp) {
    int tok;
    int32_t blk;
    if constexpr (SEL) {
      blk = selected(P, b, g, blk_beg + tid, L, tok);
    } else {
      blk = P.tables[static_cast<int64_t>(b) * P.max_blocks + blk_beg + tid];
      tok = min(kT, L - (blk_beg + tid) * kT);
    }
    // a block outside the pool counts as if it were not in the context
    const bool ok = blk >= 0 && blk < P.nb;
    row[tid] = ok ? blk : 0;
    s_tok[tid] = ok ? tok : 0;
  }
  // queries: column r is head r % G, dims 32 qd + 8 s .. + 7 in operand s
  u32x4 bq[4];
  {
    const int j = r % G;
    const uint4* q = reinterpret_cast<const uint4*>(
        P.q + (static_cast<int64_t>(b) * P.Hq + g * G + j) * kD + 32 * qd);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const uint4 u = q[s];
      bq[s] = u32x4{u.x, u.y, u.z, u.w};
    }
  }
  const int copy = r / G;  // which part of the probabilities this column takes
  __syncthreads();

  const uint32_t first_host = static_cast<uint32_t>(P.host_from >> 21);
  auto fetch = [&](int i, Block4& x) {
    x.k = x.v = x.vs = u32x4{0, 0, 0, 0};
    x.ks = 0;
    x.tok = 0;
    if (i >= nbp) return;  // uniform over the wavefront
    x.tok = __builtin_amdgcn_readfirstlane(s_tok[i]);
    if (x.tok == 0) return;
    const bst::Fp4At at = bst::fp4_at(g, __builtin_amdgcn_readfirstlane(row[i]), P.nb);
    const bool host = at.page >= first_host;
    const uint64_t off = static_cast<uint64_t>(host ? at.page - first_host : at.page) << 21;
    const char* const pk = (host ? P.k_host : P.k_hbm) + off;
    const char* const pv = (host ? P.v_host : P.v_hbm) + off;
    const uint32_t code = at.idx * bst::kFp4Code, sc = bst::kFp4ScaleAt + at.idx * bst::kFp4Scale;
    x.k = *reinterpret_cast<const u32x4*>(pk + code + r * 64 + qd * 16);
    x.ks = *reinterpret_cast<const uint8_t*>(pk + sc + r * 4 + qd);
    x.v = *reinterpret_cast<const u32x4*>(pv + code + lane * 16);
    x.vs = *reinterpret_cast<const u32x4*>(pv + sc + qd * 16);
  };
  const float sc2 = P.scale * 1.4426950408889634f;  // log2(e)
  // a block's scores in the log2 domain: -inf for tokens that do not count
  auto scores = [&](const Block4& x) {
    const float ks = bst::fp4_scale(x.ks);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 a = {fp4_unpack<0>(x.k[i], ks), fp4_unpack<1>(x.k[i], ks),
                       fp4_unpack<2>(x.k[i], ks), fp4_unpack<3>(x.k[i], ks)};
      s = mfma(a, bq[i], s);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = 4 * qd + i < x.tok ? s[i] * sc2 : -INFINITY;
    return s;
  };
  // V^T of the 16-dim tiles 2 g, 2 g + 1: four tokens of the lane's dim,
  // packed in pairs (a token that does not count is left out by a finite
  // scale, since its probability 0 must not meet a NaN)
  auto values = [&](const Block4& x, uint32_t (*t)[2]) {
    u32x4 vs = x.vs;
#pragma unroll
    for (int i = 0; i < 4; ++i) vs[i] = 4 * qd + i < x.tok ? vs[i] : 0;
    auto tile = [&](auto sel, int gr) {
      constexpr int SELB = decltype(sel)::value;
      uint32_t c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // the scale byte moved to the exponent; the bits around it do not count
        const uint32_t e = SELB == 0 ? vs[i] << 23 : SELB == 1 ? vs[i] << 15
                           : SELB == 2 ? vs[i] << 7 : vs[i] >> 1;
        c[i] = fp4_unpack<SELB>(x.v[i], __uint_as_float(e));
      }
      t[2 * gr][0] = __builtin_amdgcn_perm(c[1], c[0], 0x05040100);
      t[2 * gr][1] = __builtin_amdgcn_perm(c[3], c[2], 0x05040100);
      t[2 * gr + 1][0] = __builtin_amdgcn_perm(c[1], c[0], 0x07060302);
      t[2 * gr + 1][1] = __builtin_amdgcn_perm(c[3], c[2], 0x07060302);
    };
    tile(std::integral_constant<int, 0>{}, 0);
    tile(std::integral_constant<int, 1>{}, 1);
    tile(std::integral_constant<int, 2>{}, 2);
    tile(std::integral_constant<int, 3>{}, 3);
  };
  // this column's part of a probability
  auto share = [&](float p) {
    const float p0 = __uint_as_float(__float_as_uint(p) & 0xffff0000u);
    if constexpr (PARTS == 2) return copy == 0 ? p0 : p - p0;
    const float p1 = p - p0, p10 = __uint_as_float(__float_as_uint(p1) & 0xffff0000u);
    return copy == 0 ? p0 : copy == 1 ? p10 : p1 - p10;
  };
  auto pack = [&](float lo, float hi) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    return __builtin_bit_cast(uint32_t,
                              __builtin_convertvector(f32x2{lo, hi}, bst::bf16x2));
  };

  float m = -INFINITY, l = 0.f;
  f32x4 acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int i = 2 * wave; i < nbp; i += 8) {
    Block4 x0, x1;
    fetch(i, x0);
    fetch(i + 1, x1);
    const f32x4 s0 = scores(x0), s1 = scores(x1);
    float mc = m;
#pragma unroll
    for (int e = 0; e < 4; ++e) mc = fmaxf(mc, fmaxf(s0[e], s1[e]));
    mc = col_max(mc);
    if (__any(mc > m)) {
      const float c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mc);
      l *= c;
#pragma unroll
      for (int t = 0; t < 8; ++t) acc[t] *= c;
      m = mc;
    }
    float p[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // -inf: a token that does not count (also where the maximum still is -inf)
      p[e] = s0[e] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s0[e] - m);
      p[4 + e] = s1[e] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s1[e] - m);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) l += p[e];
    u32x4 bp;
#pragma unroll
    for (int e = 0; e < 4; ++e) bp[e] = pack(share(p[2 * e]), share(p[2 * e + 1]));
    uint32_t t0[8][2], t1[8][2];
    values(x0, t0);
    values(x1, t1);
#pragma unroll
    for (int t = 0; t < 8; ++t)
      acc[t] = mfma(u32x4{t0[t][0], t0[t][1], t1[t][0], t1[t][1]}, bp, acc[t]);
  }
  l = col_sum(l);
  if (r < PARTS * G) {
#pragma unroll
    for (int t = 0; t < 8; ++t)
      *reinterpret_cast<f32x4*>(&s_acc[wave][r][16 * t + 4 * qd]) = acc[t];
    if (qd == 0) {
      s_ml[wave][r][0] = m;
      s_ml[wave][r][1] = l;
    }
  }
  __syncthreads();
  // four dims of a head per thread: the wavefronts in order, each one's parts
  // from the largest, at the common maximum
  for (int e = tid; e < G * (kD / 4); e += kThreads) {
    const int j = e / (kD / 4), d4 = e % (kD / 4) * 4;
    float M = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, s_ml[w][j][0]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mw = s_ml[w][j][0];
      const float c = mw == M ? 1.f : __builtin_amdgcn_exp2f(mw - M);
      sum += s_ml[w][j][1] * c;
      f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < PARTS; ++u)
        a += *reinterpret_cast<const f32x4*>(&s_acc[w][u * G + j][d4]);
      o += a * c;
    }
    const int64_t at = (static_cast<int64_t>(b) * P.Hq + g * G + j) * P.max_parts + part;
    *reinterpret_cast<f32x4*>(P.part_acc + at * kD + d4) = o;
    if (d4 == 0) {
      P.part_ml[at * 2] = sum == sum ? M : 0.f;  // NaN must not look empty to the merge
      P.part_ml[at * 2 + 1] = sum;
    }
  }
}

template <int PARTS, bool SEL>
void launch(const AttnParams& P, unsigned grid, hipStream_t s) {
  if (P.B <= 64)
    hipLaunchKernelGGL((attn4_partition<PARTS, true, SEL>), dim3(grid), dim3(kThreads), 0, s, P);
  else
    hipLaunchKernelGGL((attn4_partition<PARTS, false, SEL>), dim3(grid), dim3(kThreads), 0, s, P);
}

}  // namespace

namespace bst {
namespace attn {

int launch_fp4(AttnParams& P, hipStream_t s) {
  const int64_t grid = static_cast<int64_t>(P.H) * P.B * P.n_parts;
  if (grid > 0x7fffffff) return fail(BOOST_EINVAL, "grid too large");
  const unsigned n = static_cast<unsigned>(grid);
  if (P.Hq / P.H <= 5)
    P.sel ? launch<3, true>(P, n, s) : launch<3, false>(P, n, s);
  else
    P.sel ? launch<2, true>(P, n, s) : launch<2, false>(P, n, s);
  BOOST_HIP(hipGetLastError());
  return BOOST_OK;
}

}  // namespace attn
}  // namespace bst
