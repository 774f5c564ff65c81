// Formats of a KV pool's head-blocks (16 tokens of one KV head of K or V) and
// the 4-bit conversions, shared by the kernels that touch the pool.
//
// BOOST_KV_BF16: [T][D] bf16, whole head-blocks one after another in a page.
//
// BOOST_KV_FP4 (D = 128): a token's 128 values are four groups of 32
// consecutive dims; a group holds E2M1 codes (0, 1/2, 1, 3/2, 2, 3, 4, 6 and
// their negatives) times a power of two 2^e, kept as the byte e + 127.  e is
// the smallest with max|x| <= 7 * 2^e, so no value is off by more than half
// the step around it (from 6 on, the step is the 2 below it), clamped to
// [-127, 125] (codes times 2^125 stay finite in bf16); 255 stands for a group
// with an infinity or a NaN, all of whose values read back as NaN.  A page
// holds kFp4Page head-blocks: their 1024 code bytes first, then their 64
// scale bytes, so a page's tier is the tier of all that belongs to its blocks.
//
//   K codes  [group][token][16 bytes], the even dim in the low nibble: what one
//            lane of a matrix-core operand holds (row = token), the lanes of a
//            wavefront one after another (64 bytes apart, a head-block took
//            twice the cache accesses).
//   V codes  [token / 4][r][token % 4]: the dword of dims 8 r .. 8 r + 7, so
//            the 16 bytes at 256 * (token / 4) + 16 * r are what one lane
//            holds of the transposed operand: four tokens of eight dims that
//            share a scale.  A token's bytes are its own: two tokens are
//            written at once without a race.
//   scales   K [group][token]; V [token / 4][group][token % 4], the four of
//            such a lane in one dword.
#pragma once
#include <hip/hip_runtime.h>

#include "runtime.h"

namespace bst {

constexpr int kFp4D = 128;                                   // head dimension
constexpr int kFp4Tok = 16;                                  // tokens per block
constexpr uint32_t kFp4Code = kFp4Tok * kFp4D / 2;           // code bytes of a head-block
constexpr uint32_t kFp4Scale = kFp4Tok * kFp4D / 32;         // scale bytes
constexpr uint32_t kFp4Page = 1920;                          // head-blocks per page
constexpr uint32_t kFp4ScaleAt = kFp4Page * kFp4Code;        // scales' offset in a page
static_assert(kFp4Page * (kFp4Code + kFp4Scale) <= kPage, "4-bit head-blocks of a page");

// Place of head-block (head, block) of a 4-bit tensor: page and index in it.
struct Fp4At {
  uint32_t page, idx;
};
__device__ __forceinline__ Fp4At fp4_at(int head, int block, int nb) {
  const uint32_t b = static_cast<uint32_t>(block);
  return {static_cast<uint32_t>(head) * (static_cast<uint32_t>(nb) / kFp4Page) + b / kFp4Page,
          b % kFp4Page};
}

// Scale byte of a group whose largest magnitude is amax (a bf16 value, given
// by its fp32 bits without the sign).  With amax = 2^E (1 + m / 128):
// e = E - 2, one more where 4 (1 + m / 128) > 7, that is m > 96.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t amax_bits) {
  const int f = static_cast<int>(amax_bits >> 23);  // E + 127
  if (f == 255) return 255;
  const int m = static_cast<int>((amax_bits >> 16) & 127);
  return static_cast<uint32_t>(min(max(f - 2 + (m > 96), 0), 252));
}

// The fp32 scale operand of the conversions; they use its exponent alone, so
// byte 0 (exponent field 0) is 2^-127 and 255 gives NaN.
__device__ __forceinline__ float fp4_scale(uint32_t byte) {
  return __uint_as_float(byte << 23);
}

// Byte offset of a token's scale of group g among a head-block's 64.
__device__ __forceinline__ uint32_t fp4_k_scale_at(int tok, int g) { return g * 16 + tok; }
__device__ __forceinline__ uint32_t fp4_v_scale_at(int tok, int g) {
  return (tok / 4) * 16 + g * 4 + tok % 4;
}
// ... of its K codes of group g, and of its V codes' dword r.
__device__ __forceinline__ uint32_t fp4_k_code_at(int tok, int g) { return g * 256 + tok * 16; }
__device__ __forceinline__ uint32_t fp4_v_code_at(int tok, int r) {
  return (tok / 4) * 256 + r * 16 + (tok % 4) * 4;
}

// Codes of a (low nibble) and b (high nibble): round to nearest, ties to the
// even code, saturating.  Byte SEL of old is replaced.
template <int SEL>
__device__ __forceinline__ uint32_t fp4_pack(uint32_t old, float a, float b, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, scale, SEL);
}

// Two bf16 values (low half: low nibble) of byte SEL of codes.
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
template <int SEL>
__device__ __forceinline__ uint32_t fp4_unpack(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t,
                            __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}

}  // namespace bst
