// a5 over a 4-bit pool: GQA paged-attention decode whose K and V are E2M1
// codes with a power-of-two scale per token and 32 dims (kvfmt.h).
//
// Work items and partitions are those of the bf16 kernel (attn_items.h); a
// context of one partition is finished by its workgroup, the others leave
// partial sums for the merge.  Within an item every wavefront takes pairs of
// blocks (32 tokens) in turn, on the matrix cores:
//
//   scores  S[t, c] = sum_d K[t, d] q[c, d], one 16x16x32 product per 8 dims
//           of each group: lane (r, qd) holds token r's codes of group qd, one
//           16-byte load, converted to bf16 with the group's scale (exact: a
//           code has two significant bits, the scale is a power of two).  q is
//           bf16, so every product is exact and the sum is fp32.
//   softmax the result leaves tokens 4 qd .. 4 qd + 3 of column c in a lane;
//           running maximum and sum per column in fp32.
//   output  O[d, c] = sum_t V[t, d] p[t, c]: the probabilities stay in the
//           lanes that computed them, because the sum over t may run in any
//           order as long as V's operand follows it: lane (r, qd) holds tokens
//           4 qd .. 4 qd + 3 of dims 8 r .. 8 r + 7, again one 16-byte load.
//           A conversion gives two neighbouring dims of one token, where an
//           operand register wants two terms of the sum: they are taken as two
//           terms, and a column's register holds (p, 0) or (0, p), so that it
//           sums the even dims alone or the odd ones.  No value is moved.
//
// Bound by the bytes where there are many (64 requests, 160 MB in 1 KiB pieces:
// 32 us, 5.0 TB/s, without the merge), by the chain length, block ids, codes
// where there are few (one request of 301 tokens: 4.9 us).
//
// Columns: a call has G = Hq / H query heads to 16 columns.  Up to four heads,
// column c is head c % 4, odd or even dims by bit 2, and by bit 3 one of two
// parts of the fp32 probability: its first 8 significant bits, or the rest
// rounded to 8.  Up to eight heads, bit 3 is odd or even, and the parts are two
// products into the same sums.  Either way p enters with 16 to 17 bits, an
// error of 2^-17 of each p at most, below what fp32 scores of 128 products
// carry.
#include <cmath>
#include <type_traits>

#include "attn_items.h"
#include "kvfmt.h"

namespace {

using namespace bst::attn;
using bst::fp4_unpack;

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr float kLowest = 3.402823466e+38f;
constexpr int kAccRow = kD + 4;  // floats of a head's row in LDS (banks)

__device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// v of the four lanes that hold one column (16 and 32 lanes apart) by F, the
// same bits in each of them.
template <typename F>
__device__ __forceinline__ float over_column(float v, F f) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t w = __float_as_uint(f(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// One block's codes and scales in a lane.
struct Block4 {
  u32x4 k, v;   // 32 codes of token r, group qd; four tokens of dims 8 r ..
  uint32_t ks;  // scale byte of token r, group qd
  uint32_t vs;  // scale bytes of tokens 4 qd .., group r / 4
  int tok;      // tokens that count
};

// EIGHT: more than four query heads per KV head.  W wavefronts (kWave and
// kGroup, the searches: 4).  kEach: see item_each.
enum class Items { kWave, kGroup, kEach };
template <bool EIGHT, Items ITEMS, bool SEL, int W>
__global__ __launch_bounds__(64 * W) void attn4_partition(AttnParams P) {
  static_assert(ITEMS == Items::kEach || 64 * W == kThreads, "item search");
  __shared__ float s_acc[W][8][kAccRow];  // heads (EIGHT), else 4 heads of each part
  __shared__ float s_ml[W][8][2];
  __shared__ int32_t row[kMaxPartBlocks];    // the partition's pool blocks
  __shared__ int32_t s_tok[kMaxPartBlocks];  // and their tokens that count
  __shared__ int s_red[4], s_pick[5];
  int part, b, g, L;
  if constexpr (ITEMS == Items::kWave) {
    if (!item_of_wave(P, blockIdx.x, b, g, part, L)) return;  // uniform
  } else if constexpr (ITEMS == Items::kGroup) {
    if (!item_of(P, blockIdx.x, b, g, part, L, s_red, row, s_pick)) return;  // uniform
    __syncthreads();  // row has served the search
  } else {
    item_each(P, b, g, part);
    L = P.lens[b];
  }
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  Listed entry;  // of a list: one a thread
  if constexpr (SEL) entry = listed(P, b, g, part, tid);
  const int r = lane & 15, qd = lane >> 4;
  const int G = P.Hq / P.H;
  const int n_blk = L <= 0 ? 0 : min(blocks_in(L), P.item_blocks);
  const int blk_beg = part * P.part_blocks;
  if (ITEMS == Items::kEach && part > 0 && blk_beg >= n_blk) return;  // uniform
  const int nbp = min(n_blk, blk_beg + P.part_blocks) - blk_beg;
  const bool whole = n_blk <= P.part_blocks;
  static_assert(!SEL || 64 * W >= kMaxPartBlocks, "a thread an entry");
  for (int i = tid; i < nbp; i += 64 * W) {
    int tok;
    int32_t blk;
    if constexpr (SEL) {
      blk = selected(P, entry, L, tok);
    } else {
      blk = P.tables[static_cast<int64_t>(b) * P.max_blocks + blk_beg + i];
      tok = min(kT, L - (blk_beg + i) * kT);
    }
    // a block outside the pool counts as if it were not in the context
    const bool ok = blk >= 0 && blk < P.nb;
    row[i] = ok ? blk : 0;
    s_tok[i] = ok ? tok : 0;
  }
  constexpr int kHeads = EIGHT ? 8 : 4;
  const int head = r % kHeads;  // this column's, if below G
  const bool odd = r & kHeads;  // odd dims
  const bool rest = !EIGHT && (r & 8);  // the second part of p
  // queries: dims 32 qd + 8 s .. + 7 in operand s
  u32x4 bq[4];
  {
    const uint4* q = reinterpret_cast<const uint4*>(
        P.q + (static_cast<int64_t>(b) * P.Hq + g * G + min(head, G - 1)) * kD + 32 * qd);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const uint4 u = q[s];
      bq[s] = u32x4{u.x, u.y, u.z, u.w};
    }
  }
  const uint32_t code_off = lane * 16, ks_off = lane, vs_off = bst::fp4_v_scale_at(4 * qd, r / 4);
  __syncthreads();

  const uint32_t first_host = static_cast<uint32_t>(P.host_from >> 21);
  // Block i of the partition; past its end the last one with no token that
  // counts, so that loads need no branch (a block outside the pool: block 0).
  auto fetch = [&](int i, Block4& x) {
    const int at_i = min(i, nbp - 1);
    const int tok = __builtin_amdgcn_readfirstlane(s_tok[at_i]);
    x.tok = i < nbp ? tok : 0;
    const bst::Fp4At at = bst::fp4_at(g, __builtin_amdgcn_readfirstlane(row[at_i]), P.nb);
    const bool host = at.page >= first_host;
    const uint64_t off = static_cast<uint64_t>(host ? at.page - first_host : at.page) << 21;
    const char* const pk = (host ? P.k_host : P.k_hbm) + off;
    const char* const pv = (host ? P.v_host : P.v_hbm) + off;
    const uint32_t code = at.idx * bst::kFp4Code, sc = bst::kFp4ScaleAt + at.idx * bst::kFp4Scale;
    x.k = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(pk + code + code_off));
    x.ks = *reinterpret_cast<const uint8_t*>(pk + sc + ks_off);
    x.v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(pv + code + code_off));
    x.vs = *reinterpret_cast<const uint32_t*>(pv + sc + vs_off);
  };
  const float sc2 = P.scale * 1.4426950408889634f;  // log2(e)
  auto scores = [&](const Block4& x) {
    const float ks = bst::fp4_scale(x.ks);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 a = {fp4_unpack<0>(x.k[i], ks), fp4_unpack<1>(x.k[i], ks),
                       fp4_unpack<2>(x.k[i], ks), fp4_unpack<3>(x.k[i], ks)};
      s = mfma(a, bq[i], s);
    }
    return s;
  };
  // dims 8 r + 2 B, + 1 of the lane's four tokens; the scale byte is moved to
  // the exponent, the bits around it do not count
  auto values = [&](const Block4& x, auto byte) {
    constexpr int B = decltype(byte)::value;
    return u32x4{fp4_unpack<B>(x.v[0], __uint_as_float(x.vs << 23)),
                 fp4_unpack<B>(x.v[1], __uint_as_float(x.vs << 15)),
                 fp4_unpack<B>(x.v[2], __uint_as_float(x.vs << 7)),
                 fp4_unpack<B>(x.v[3], __uint_as_float(x.vs >> 1))};
  };
  // A probability's part for this column: its first 16 bits, in the lower or
  // the upper half of the register by place, or the rest of them.
  const uint32_t place = odd ? 0x07060c0cu : 0x0c0c0706u;  // 0x0c: a zero byte
  auto first = [&](float p) { return __builtin_amdgcn_perm(__float_as_uint(p), 0u, place); };
  auto second = [&](float p) {
    const float x = p - __uint_as_float(__float_as_uint(p) & 0xffff0000u);
    return __builtin_amdgcn_perm(__float_as_uint(x) + 0x8000u, 0u, place);
  };
  // without a branch over the columns: the mask is all ones in the columns of
  // the second part
  const uint32_t off = rest ? 0xffff0000u : 0u, round = rest ? 0x8000u : 0u;
  auto either = [&](float p) {
    const float x = p - __uint_as_float(__float_as_uint(p) & off);
    return __builtin_amdgcn_perm(__float_as_uint(x) + round, 0u, place);
  };

  // m starts at the lowest finite value: exp2(-inf - m) is 0 from the first
  // token on, also while none has counted
  float m = -kLowest, l = 0.f;
  f32x4 acc[4];  // dims 8 (4 qd + i) + 2 byte + odd
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto consume = [&](Block4& x0, Block4& x1) {
    f32x4 s0 = scores(x0), s1 = scores(x1);
    if (x0.tok + x1.tok < 2 * kT) {  // uniform: some tokens do not count
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in0 = 4 * qd + e < x0.tok, in1 = 4 * qd + e < x1.tok;
        s0[e] = in0 ? s0[e] : -INFINITY;
        s1[e] = in1 ? s1[e] : -INFINITY;
        // their probability 0 must not meet a NaN: a finite scale
        x0.vs &= in0 ? ~0u : ~(255u << (8 * e));
        x1.vs &= in1 ? ~0u : ~(255u << (8 * e));
      }
    }
    float mc = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])),
                     fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
    mc = fmaxf(m, over_column(mc, [](float a, float b) { return fmaxf(a, b); }));
    if (__any(mc > m)) {
      const float c = __builtin_amdgcn_exp2f((m - mc) * sc2);
      l *= c;
#pragma unroll
      for (int t = 0; t < 4; ++t) acc[t] *= c;
      m = mc;
    }
    float p[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // (the difference first: the largest score has weight 1 at any size)
      p[e] = __builtin_amdgcn_exp2f((s0[e] - m) * sc2);
      p[4 + e] = __builtin_amdgcn_exp2f((s1[e] - m) * sc2);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) l += p[e];
    u32x4 b0, b1, c0, c1;  // the parts of p (EIGHT: the second in c)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (EIGHT) {
        b0[e] = first(p[e]);
        b1[e] = first(p[4 + e]);
        c0[e] = second(p[e]);
        c1[e] = second(p[4 + e]);
      } else {
        b0[e] = either(p[e]);
        b1[e] = either(p[4 + e]);
      }
    }
    auto tile = [&](auto byte) {
      constexpr int B = decltype(byte)::value;
      const u32x4 v0 = values(x0, byte), v1 = values(x1, byte);
      acc[B] = mfma(v0, b0, acc[B]);
      acc[B] = mfma(v1, b1, acc[B]);
      if constexpr (EIGHT) {
        acc[B] = mfma(v0, c0, acc[B]);
        acc[B] = mfma(v1, c1, acc[B]);
      }
    };
    tile(std::integral_constant<int, 0>{});
    tile(std::integral_constant<int, 1>{});
    tile(std::integral_constant<int, 2>{});
    tile(std::integral_constant<int, 3>{});
  };
  if (nbp > 0) {
    // The next pair's loads are out while a pair is computed.  They are issued
    // without a branch (past the end: the last block again, from the caches),
    // so that the waits can count them.
    constexpr int kStep = 2 * W;
    Block4 a0, a1, b0, b1;
    fetch(2 * wave, a0);
    fetch(2 * wave + 1, a1);
    for (int i = 2 * wave; i < nbp; i += 2 * kStep) {
      fetch(i + kStep, b0);
      fetch(i + kStep + 1, b1);
      consume(a0, a1);
      if (i + kStep >= nbp) break;  // uniform over the wavefront
      fetch(i + 2 * kStep, a0);
      fetch(i + 2 * kStep + 1, a1);
      consume(b0, b1);
    }
  }
  l = over_column(l, [](float a, float b) { return a + b; });
  {
    float* const to = &s_acc[wave][EIGHT ? head : head + (rest ? 4 : 0)][32 * qd + (odd ? 1 : 0)];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < 4; ++t) to[8 * i + 2 * t] = acc[t][i];
    if (lane < kHeads) {
      s_ml[wave][lane][0] = m;
      s_ml[wave][lane][1] = l;
    }
  }
  __syncthreads();
  // four dims of a head per thread: the wavefronts in order, each one's parts
  // from the largest, at the common maximum
  for (int e = tid; e < G * (kD / 4); e += 64 * W) {
    const int j = e / (kD / 4), d4 = e % (kD / 4) * 4;
    float M = -kLowest, sum = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, s_ml[w][j][0]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float c = __builtin_amdgcn_exp2f((s_ml[w][j][0] - M) * sc2);
      sum += s_ml[w][j][1] * c;
      f32x4 a = *reinterpret_cast<const f32x4*>(&s_acc[w][j][d4]);
      if constexpr (!EIGHT) a += *reinterpret_cast<const f32x4*>(&s_acc[w][j + 4][d4]);
      o += a * c;
    }
    const int64_t out = static_cast<int64_t>(b) * P.Hq + g * G + j;
    if (whole) {  // uniform
      const float inv = sum != 0.f ? 1.f / sum : 0.f;  // nothing counted: a zero row
      o *= inv;
      if (P.out_bf16) {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(P.out) + out * kD + d4) =
            make_uint2(to_bf16(o[0]) | static_cast<uint32_t>(to_bf16(o[1])) << 16,
                       to_bf16(o[2]) | static_cast<uint32_t>(to_bf16(o[3])) << 16);
      } else {
        float* const to = static_cast<float*>(P.out) + out * kD + d4;
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = o[i];
      }
      continue;
    }
    const int64_t at = out * P.max_parts + part;
    *reinterpret_cast<f32x4*>(P.part_acc + at * kD + d4) = o;
    if (d4 == 0) {
      // nothing counted: what the merge takes for empty (a NaN is not)
      P.part_ml[at * 2] = sum == 0.f ? -INFINITY : M;
      P.part_ml[at * 2 + 1] = sum;
    }
  }
}

template <bool EIGHT>
void launch(const AttnParams& P, dim3 grid, int n_cu, hipStream_t s) {
  auto go = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, P);
  };
  // a workgroup alone on its compute unit: a pair is one chain of products,
  // maximum, exponentials and products, 83 ns a block with four wavefronts,
  // 61 with eight (57 with 16: the unit's bandwidth); 32 requests of 1500
  // tokens 12.4 us with eight and 13.9 with four, 64 of 1000 17.2 and 15.9
  const bool alone = P.n_parts == 1 && P.B * P.H <= n_cu;
  if (P.sel && alone)
    go(attn4_partition<EIGHT, Items::kEach, true, 8>, 512);
  else if (P.sel)
    go(attn4_partition<EIGHT, Items::kEach, true, 4>, 256);
  else if (alone)
    go(attn4_partition<EIGHT, Items::kEach, false, 8>, 512);
  else if (P.n_parts == 1)
    go(attn4_partition<EIGHT, Items::kEach, false, 4>, 256);
  else if (P.B <= 64)
    go(attn4_partition<EIGHT, Items::kWave, false, 4>, 256);
  else
    go(attn4_partition<EIGHT, Items::kGroup, false, 4>, 256);
}

}  // namespace

namespace bst {
namespace attn {

int launch_fp4(AttnParams& P, int n_cu, hipStream_t s) {
  const int64_t grid = static_cast<int64_t>(P.H) * P.B * P.n_parts;
  dim3 g(static_cast<unsigned>(grid));
  if (grid > 0x7fffffff || ((P.sel || P.n_parts == 1) && !grid_each(P, g)))
    return fail(BOOST_EINVAL, "grid too large");
  if (P.Hq / P.H <= 4)
    launch<false>(P, g, n_cu, s);
  else
    launch<true>(P, g, n_cu, s);
  BOOST_HIP(hipGetLastError());
  return BOOST_OK;
}

}  // namespace attn
}  // namespace bst
