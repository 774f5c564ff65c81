// KV pool (§4.2 LPP, §4.5 heads-outermost layout and two free lists) and the
// kernels that write its tokens and read them back.  Every layer has a K and
// a V tensor [H][NB][T][D], bf16 or in 4 bits (kvfmt.h); the LPP tail pages of
// each tensor live in pinned host memory, the rest in one HBM slab; the device
// page table maps (layer, K/V, page) to an address.
#include <algorithm>
#include <cstring>
#include <exception>
#include <new>
#include <type_traits>

#include "kvfmt.h"
#include "runtime.h"

namespace {

constexpr int kPartTokensMin = 64;  // smallest attention partition (4 blocks)

// One lane per 16 bytes of one (token, head) row of K and of V.
__global__ __launch_bounds__(256) void kv_write_kernel(
    const char* const* __restrict__ pt_k, const char* const* __restrict__ pt_v,
    const int32_t* __restrict__ slots, const uint4* __restrict__ k,
    const uint4* __restrict__ v, int n, int H, int D, int T, int nb) {
  const int chunks = D / 8;  // 16-byte chunks per head row
  const int64_t t = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t total = static_cast<int64_t>(n) * H * chunks;
  if (t >= total) return;
  const int c = static_cast<int>(t % chunks);
  const int64_t th = t / chunks;  // token * H + head
  const int h = static_cast<int>(th % H);
  const int64_t i = th / H;
  const int32_t slot = slots[i];
  if (slot < 0 || slot >= static_cast<int64_t>(nb) * T) return;
  const int32_t blk = slot / T, off = slot % T;
  const uint64_t byte = ((static_cast<uint64_t>(h) * nb + blk) * T + off) * D * 2 +
                        static_cast<uint64_t>(c) * 16;
  const uint64_t page = byte >> 21, in = byte & (bst::kPage - 1);
  *reinterpret_cast<uint4*>(const_cast<char*>(pt_k[page]) + in) = k[t];
  *reinterpret_cast<uint4*>(const_cast<char*>(pt_v[page]) + in) = v[t];
}

// Reads token slots back: the inverse of kv_write_kernel.
__global__ __launch_bounds__(256) void kv_read_kernel(
    const char* const* __restrict__ pt_k, const char* const* __restrict__ pt_v,
    const int32_t* __restrict__ slots, uint4* __restrict__ k, uint4* __restrict__ v, int n, int H,
    int D, int T, int nb) {
  const int chunks = D / 8;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (t >= static_cast<int64_t>(n) * H * chunks) return;
  const int c = static_cast<int>(t % chunks);
  const int64_t th = t / chunks;
  const int h = static_cast<int>(th % H);
  const int32_t slot = slots[th / H];
  if (slot < 0 || slot >= static_cast<int64_t>(nb) * T) return;
  const uint64_t byte = ((static_cast<uint64_t>(h) * nb + slot / T) * T + slot % T) * D * 2 +
                        static_cast<uint64_t>(c) * 16;
  const uint64_t page = byte >> 21, in = byte & (bst::kPage - 1);
  k[t] = *reinterpret_cast<const uint4*>(pt_k[page] + in);
  v[t] = *reinterpret_cast<const uint4*>(pt_v[page] + in);
}

// ---- 4 bits.  A workgroup takes 16 rows in a row (a prompt's tokens of one
// block, mostly) of one KV head, a lane 8 dims: 16 bytes in and a dword of
// codes out for K and V each, or the reverse; a quad of lanes shares a scale.
// Bound by the bytes, 512 and 136 a row: whole lines of the rows, and the
// head-block's lines put together in one L2.
constexpr int kRows4 = 16;

// 16 bytes that are read or written once, past the caches, where the pool's
// lines wait to be whole (write and read back of 20011 tokens with 8 heads, 207
// MB: 45.5 us through them, 38.4 with the reads past them, 37.6 with the writes;
// of 2000 7.5 and 6.8 with the writes, of 100000 214 and 174).
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
__device__ __forceinline__ uint4 streamed(const uint4* at) {
  const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at));
  return make_uint4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void streamed(uint4* at, const uint4& v) {
  __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(at));
}

// Slot of row i: given (slots), or that of request i's token at pos[i] (a
// position or a block outside the table or the pool: -1).
struct RowSlot {
  const int32_t* slots;
  const int32_t* tables;
  const int32_t* pos;
  int max_blocks;
};
__device__ __forceinline__ int64_t slot_of(const RowSlot& r, int64_t i, int nb) {
  int64_t slot;
  if (r.slots) {
    slot = r.slots[i];
  } else {
    const int p = r.pos[i];
    if (p < 0 || p / bst::kFp4Tok >= r.max_blocks) return -1;
    const int32_t blk = r.tables[i * r.max_blocks + p / bst::kFp4Tok];
    if (blk < 0) return -1;
    slot = static_cast<int64_t>(blk) * bst::kFp4Tok + p % bst::kFp4Tok;
  }
  return slot < static_cast<int64_t>(nb) * bst::kFp4Tok ? slot : -1;
}

// Eight bf16 values in 4 bits; sb: their group's scale byte, found over the
// quad of lanes that hold it.
__device__ __forceinline__ uint32_t codes_of(const uint4& u, uint32_t& sb) {
  using namespace bst;
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    amax = max(amax, max((w[i] << 16) & 0x7fff0000u, w[i] & 0x7fff0000u));
  auto far = [&](auto ctrl) {
    return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(
        static_cast<int>(amax), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  amax = max(amax, far(std::integral_constant<int, 0xb1>{}));  // the lane xor 1
  amax = max(amax, far(std::integral_constant<int, 0x4e>{}));  // xor 2
  sb = fp4_scale_byte(amax);
  const float s = fp4_scale(sb);
  auto lo = [&](int i) { return __uint_as_float(w[i] << 16); };
  auto hi = [&](int i) { return __uint_as_float(w[i] & 0xffff0000u); };
  uint32_t c = fp4_pack<0>(0u, lo(0), hi(0), s);
  c = fp4_pack<1>(c, lo(1), hi(1), s);
  c = fp4_pack<2>(c, lo(2), hi(2), s);
  return fp4_pack<3>(c, lo(3), hi(3), s);
}

// ... and back.
__device__ __forceinline__ uint4 values_of(uint32_t c, uint32_t sb) {
  using namespace bst;
  const float s = fp4_scale(sb);
  return make_uint4(fp4_unpack<0>(c, s), fp4_unpack<1>(c, s), fp4_unpack<2>(c, s),
                    fp4_unpack<3>(c, s));
}

// Where lane r (of 16) of a row finds its dwords and scales.
struct Row4 {
  char *k, *v, *ks, *vs;
};
__device__ __forceinline__ Row4 row4(const char* const* pt_k, const char* const* pt_v,
                                     int64_t slot, int h, int nb, int r) {
  using namespace bst;
  const int tok = static_cast<int>(slot % kFp4Tok);
  const Fp4At at = fp4_at(h, static_cast<int>(slot / kFp4Tok), nb);
  char* const pk = const_cast<char*>(pt_k[at.page]);
  char* const pv = const_cast<char*>(pt_v[at.page]);
  const uint32_t code = at.idx * kFp4Code, scale = kFp4ScaleAt + at.idx * kFp4Scale;
  return {pk + code + fp4_k_code_at(tok, r / 4) + r % 4 * 4, pv + code + fp4_v_code_at(tok, r),
          pk + scale + fp4_k_scale_at(tok, r / 4), pv + scale + fp4_v_scale_at(tok, r / 4)};
}

__global__ __launch_bounds__(16 * kRows4) void kv_write4_kernel(
    const char* const* __restrict__ pt_k, const char* const* __restrict__ pt_v, RowSlot rows,
    const uint4* __restrict__ k, const uint4* __restrict__ v, int n, int H, int nb) {
  const int r = threadIdx.x & 15, h = blockIdx.x % H;
  const int64_t i = static_cast<int64_t>(blockIdx.x / H) * kRows4 + (threadIdx.x >> 4);
  if (i >= n) return;  // whole rows of lanes
  const int64_t slot = slot_of(rows, i, nb);
  if (slot < 0) return;
  const int64_t at = (i * H + h) * 16 + r;
  const uint4 uk = streamed(k + at), uv = streamed(v + at);
  const Row4 to = row4(pt_k, pt_v, slot, h, nb, r);
  uint32_t sk, sv;
  const uint32_t ck = codes_of(uk, sk), cv = codes_of(uv, sv);
  *reinterpret_cast<uint32_t*>(to.k) = ck;
  *reinterpret_cast<uint32_t*>(to.v) = cv;
  if (r % 4 == 0) {
    *to.ks = static_cast<char>(sk);
    *to.vs = static_cast<char>(sv);
  }
}

__global__ __launch_bounds__(16 * kRows4) void kv_read4_kernel(
    const char* const* __restrict__ pt_k, const char* const* __restrict__ pt_v,
    const int32_t* __restrict__ slots, uint4* __restrict__ k, uint4* __restrict__ v, int n, int H,
    int nb) {
  const int r = threadIdx.x & 15, h = blockIdx.x % H;
  const int64_t i = static_cast<int64_t>(blockIdx.x / H) * kRows4 + (threadIdx.x >> 4);
  if (i >= n) return;
  const int64_t slot = slot_of(RowSlot{slots, nullptr, nullptr, 0}, i, nb);
  if (slot < 0) return;
  const int64_t at = (i * H + h) * 16 + r;
  const Row4 from = row4(pt_k, pt_v, slot, h, nb, r);
  const uint32_t ck = *reinterpret_cast<const uint32_t*>(from.k);
  const uint32_t cv = *reinterpret_cast<const uint32_t*>(from.v);
  const uint32_t sk = static_cast<uint8_t>(*from.ks), sv = static_cast<uint8_t>(*from.vs);
  streamed(k + at, values_of(ck, sk));
  streamed(v + at, values_of(cv, sv));
}

// Blocks copied within the pool: one workgroup (4 bits: wavefront) per (pair,
// KV head of K or V, layer), and per (pair, KV head's summary, layer) where the
// pool has summaries.  Read once and written once, past the caches: bound by
// the bytes (61 blocks of 8 heads in 32 layers, bf16 44.5 us, 5.7 TB/s;
// through the caches 52.0, with reads past them too 49.0; 200 blocks 119, 134
// and 144.  4 bits: 61 blocks 15.4 us, by workgroups 19.2, through the caches
// 21.3).
// Pairs per launch: they travel as an argument, whose every byte the host
// writes at each launch (a call for one pair: 4.0 us with room for 16, 4.5 with
// room for 448).
constexpr int kCopyFew = 16, kCopyPairs = 448;
template <int N>
struct CopyPairs {
  int32_t src[N], dst[N];
};
struct CopyParams {
  const char* const* table;  // the pool's pages [layers][2][pages]
  uint64_t pages;
  int8_t* index;             // summaries and exponents, or null
  uint64_t index_blocks;     // layers * H * nb
  int layer0, H, nb;
  int units;                 // KV heads of K, of V and of the summaries
  uint32_t block_bytes;      // bf16: bytes of a head-block
};

template <bool FP4, int N>
__global__ __launch_bounds__(256) void copy_blocks_kernel(CopyParams P, CopyPairs<N> pairs) {
  using namespace bst;
  const int s = pairs.src[blockIdx.x], d = pairs.dst[blockIdx.x];
  const int tid = FP4 ? threadIdx.x & 63 : threadIdx.x;
  const int unit = FP4 ? blockIdx.y * 4 + (threadIdx.x >> 6) : blockIdx.y;
  if (FP4 && unit >= P.units) return;
  const int which = unit / P.H, h = unit % P.H;
  const int layer = P.layer0 + static_cast<int>(blockIdx.z);
  if (which == 2) {
    const int64_t at = (static_cast<int64_t>(layer) * P.H + h) * P.nb;
    uint4* const sum = reinterpret_cast<uint4*>(P.index);
    if (tid < 16) sum[(at + d) * 16 + tid] = sum[(at + s) * 16 + tid];
    int8_t* const exp = P.index + P.index_blocks * 256;
    if (tid == 16) exp[at + d] = exp[at + s];
    return;
  }
  const char* const* pt = P.table + (2ull * layer + which) * P.pages;
  if constexpr (FP4) {
    const Fp4At a = fp4_at(h, s, P.nb), b = fp4_at(h, d, P.nb);
    const char* const from = pt[a.page];
    char* const to = const_cast<char*>(pt[b.page]);
    auto copy = [&](uint32_t dst, uint32_t src) {
      streamed(reinterpret_cast<uint4*>(to + dst), *reinterpret_cast<const uint4*>(from + src));
    };
    const uint32_t off = static_cast<uint32_t>(tid) * 16;
    copy(b.idx * kFp4Code + off, a.idx * kFp4Code + off);
    if (off < kFp4Scale)
      copy(kFp4ScaleAt + b.idx * kFp4Scale + off, kFp4ScaleAt + a.idx * kFp4Scale + off);
  } else {
    const uint64_t a = (static_cast<uint64_t>(h) * P.nb + s) * P.block_bytes;
    const uint64_t b = (static_cast<uint64_t>(h) * P.nb + d) * P.block_bytes;
    const uint32_t off = static_cast<uint32_t>(tid) * 16;
    if (off < P.block_bytes)
      streamed(reinterpret_cast<uint4*>(const_cast<char*>(pt[b >> 21]) + (b & (kPage - 1)) + off),
               *reinterpret_cast<const uint4*>(pt[a >> 21] + (a & (kPage - 1)) + off));
  }
}

// The host's exceptions end at the C entry.
template <typename F>
int guarded(F f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return bst::fail(BOOST_ENOMEM, "host memory for the allocator state");
  } catch (const std::exception& e) {
    return bst::fail(BOOST_EINVAL, "%s", e.what());
  }
}

int destroy(boost_kv_pool* p) {
  if (!p) return BOOST_OK;
  if (p->ctx && p->ctx->device >= 0) (void)hipSetDevice(p->ctx->device);
  (void)hipFree(p->d_page_table);
  (void)hipFree(p->d_part_acc);
  (void)hipFree(p->d_part_ml);
  (void)hipFree(p->d_index);
  bst::slab_free(p->hbm);
  for (auto& h : p->host) bst::slab_free(h);
  delete p;
  return BOOST_OK;
}

}  // namespace

namespace bst {
int kv_parts_for(const boost_kv_pool* p, int max_blocks) {
  const int64_t tokens = static_cast<int64_t>(max_blocks) * p->cfg.block_tokens;
  return static_cast<int>(std::max<int64_t>(1, (tokens + kPartTokensMin - 1) / kPartTokensMin));
}

int kv_device(const boost_kv_pool* p) {
  if (p->ctx->device < 0 || !p->d_page_table) return fail(BOOST_ENODEV, "plan-only pool");
  int device = -1;
  BOOST_HIP(hipGetDevice(&device));
  if (device != p->ctx->device)
    return fail(BOOST_EINVAL, "the pool is on device %d, the current one is %d", p->ctx->device,
                device);
  return BOOST_OK;
}

int kv_layer(const boost_kv_pool* p, int layer, const char* const** pk, const char* const** pv) {
  if (int rc = kv_device(p)) return rc;
  if (layer < 0 || static_cast<uint32_t>(layer) >= p->cfg.layers)
    return fail(BOOST_EINVAL, "layer %d", layer);
  *pk = p->d_page_table + (2ull * layer) * p->geom.pages;
  *pv = p->d_page_table + (2ull * layer + 1) * p->geom.pages;
  return BOOST_OK;
}

int k_pages(const boost_kv_pool* p, int layer, KPages& at) {
  const char* const *pk, * const *pv;
  if (int rc = kv_layer(p, layer, &pk, &pv)) return rc;
  const uint64_t host = p->geom.host_pages, hbm = p->geom.pages - host;
  const char* const base = p->hbm.base + 2ull * layer * hbm * kPage;
  at = {base, host ? p->host[layer].base : base, static_cast<uint32_t>(hbm)};
  return BOOST_OK;
}

int kv_write4(const boost_kv_pool* p, int layer, const int32_t* slots, const int32_t* tables,
              int max_blocks, const int32_t* positions, const void* k, const void* v, int n,
              void* stream) {
  const char* const *pk, * const *pv;
  if (int rc = kv_layer(p, layer, &pk, &pv)) return rc;
  const int H = static_cast<int>(p->cfg.kv_heads);
  const int64_t grid = (static_cast<int64_t>(n) + kRows4 - 1) / kRows4 * H;
  if (grid > 0x7fffffff) return fail(BOOST_EINVAL, "n=%d: grid too large", n);
  hipLaunchKernelGGL(kv_write4_kernel, dim3(static_cast<unsigned>(grid)), dim3(16 * kRows4), 0,
                     static_cast<hipStream_t>(stream), pk, pv,
                     RowSlot{slots, tables, positions, max_blocks}, static_cast<const uint4*>(k),
                     static_cast<const uint4*>(v), n, H, static_cast<int>(p->geom.nb));
  BOOST_HIP(hipGetLastError());
  return BOOST_OK;
}
}  // namespace bst

using namespace bst;

extern "C" {

int boost_kv_pool_create(boost_ctx* ctx, const boost_kv_cfg* cfg, boost_kv_pool** out) {
  return boost_kv_pool_create_format(ctx, cfg, BOOST_KV_BF16, out);
}

int boost_kv_pool_create_format(boost_ctx* ctx, const boost_kv_cfg* cfg, int format,
                                boost_kv_pool** out) {
  if (!ctx || !cfg || !out) return fail(BOOST_EINVAL, "null argument");
  *out = nullptr;
  if (format != BOOST_KV_BF16 && format != BOOST_KV_FP4)
    return fail(BOOST_EINVAL, "format %d", format);
  if (format == BOOST_KV_FP4 && cfg->head_dim != static_cast<uint32_t>(kFp4D))
    return fail(BOOST_EINVAL, "a 4-bit pool needs head_dim %d", kFp4D);
  if (cfg->layers == 0) return fail(BOOST_EINVAL, "0 layers");
  if (cfg->block_tokens != 16) return fail(BOOST_EINVAL, "block_tokens must be 16");
  if (cfg->head_dim != 64 && cfg->head_dim != 128)
    return fail(BOOST_EINVAL, "head_dim must be 64 or 128");
  if (cfg->kv_heads == 0) return fail(BOOST_EINVAL, "0 kv_heads");
  if (cfg->q_heads == 0 || cfg->q_heads % cfg->kv_heads || cfg->q_heads / cfg->kv_heads > 16)
    return fail(BOOST_EINVAL, "q_heads %u must be a multiple of kv_heads %u (ratio <= 16)",
                cfg->q_heads, cfg->kv_heads);
  boost_kv_pool* p = nullptr;
  try {  // host-side allocator state: per-block host heads and the two free lists
    if (fault_host_alloc()) throw std::bad_alloc();
    p = new boost_kv_pool();
    p->ctx = ctx;
    p->cfg = *cfg;
    p->format = format;
    int rc = kv_geometry(cfg->n_blocks, cfg->kv_heads, cfg->head_dim, cfg->block_tokens,
                         cfg->M, cfg->tier_mode, cfg->layers, cfg->hbm_budget_bytes,
                         format == BOOST_KV_FP4 ? kFp4Page : 0, p->geom);
    if (rc) {
      delete p;
      return rc;
    }
    p->dsr.init(p->geom);
  } catch (const std::bad_alloc&) {
    delete p;
    return fail(BOOST_ENOMEM, "KV pool: host memory for the allocator state");
  }
  int rc = BOOST_OK;
  if (ctx->device < 0) {  // plan-only: allocator bookkeeping only
    *out = p;
    return BOOST_OK;
  }
  if (cfg->max_batch == 0 || cfg->max_blocks_per_seq == 0) {
    delete p;
    return fail(BOOST_EINVAL, "max_batch and max_blocks_per_seq must be > 0");
  }
  if (hipSetDevice(ctx->device) != hipSuccess) {
    delete p;
    return fail(BOOST_EHIP, "hipSetDevice failed");
  }
  const uint64_t tensors = 2ull * cfg->layers;
  const uint64_t P = p->geom.pages, Hp = p->geom.host_pages;
  // one HBM slab for every tensor's HBM pages; the host tails in one pinned
  // slab per layer (K's tail then V's), which keeps each pinned allocation a
  // few GB even when most of a large pool lives on host
  rc = slab_alloc(ctx, tensors * (P - Hp), false, p->hbm);
  if (!rc && Hp) {
    p->host.resize(cfg->layers);
    for (uint32_t l = 0; l < cfg->layers && !rc; ++l)
      rc = slab_alloc(ctx, 2 * Hp, true, p->host[l]);
  }
  if (rc) {
    destroy(p);
    return rc;
  }
  std::vector<char*> table(tensors * P);
  for (uint64_t t = 0; t < tensors; ++t)
    for (uint64_t pg = 0; pg < P; ++pg)
      table[t * P + pg] = pg < P - Hp
                              ? p->hbm.base + (t * (P - Hp) + pg) * kPage
                              : p->host[t / 2].base + ((t % 2) * Hp + (pg - (P - Hp))) * kPage;
  p->max_parts = kv_parts_for(p, static_cast<int>(cfg->max_blocks_per_seq));
  const uint64_t rows = static_cast<uint64_t>(cfg->max_batch) * cfg->q_heads * p->max_parts;
  hipError_t e = hipMalloc(&p->d_page_table, table.size() * sizeof(char*));
  if (e == hipSuccess)
    e = hipMemcpy(p->d_page_table, table.data(), table.size() * sizeof(char*),
                  hipMemcpyHostToDevice);
  if (e == hipSuccess) e = hipMalloc(&p->d_part_acc, rows * cfg->head_dim * sizeof(float));
  if (e == hipSuccess) e = hipMalloc(&p->d_part_ml, rows * 2 * sizeof(float));
  // zero the pool so unwritten slots hold defined values
  if (e == hipSuccess && p->hbm.pages) e = hipMemset(p->hbm.base, 0, p->hbm.pages * kPage);
  for (auto& h : p->host)
    if (e == hipSuccess) std::memset(h.host_base, 0, h.pages * kPage);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    destroy(p);
    return fail(e == hipErrorOutOfMemory ? BOOST_ENOMEM : BOOST_EHIP, "KV pool: %s",
                hipGetErrorString(e));
  }
  *out = p;
  return BOOST_OK;
}

int boost_kv_pool_info(const boost_kv_pool* p, boost_kv_info* info) {
  if (!p || !info) return fail(BOOST_EINVAL, "null argument");
  info->nb_pool = p->geom.nb;
  info->blocks_per_page = p->geom.blocks_per_page;
  info->pages_per_tensor = p->geom.pages;
  info->host_pages_per_tensor = p->geom.host_pages;
  info->n_shh = p->geom.n_shh;
  info->shh_host_heads = p->geom.hi;
  info->local_host_heads = p->geom.lo;
  info->tau = p->dsr.tau();
  return BOOST_OK;
}

int boost_kv_pool_destroy(boost_kv_pool* p) { return destroy(p); }

int boost_kv_pool_format(const boost_kv_pool* p, int* format) {
  if (!p || !format) return fail(BOOST_EINVAL, "null argument");
  *format = p->format;
  return BOOST_OK;
}

int boost_kv_pages(const boost_kv_pool* p, int layer, int which, uint64_t* addresses,
                   uint64_t cap, uint64_t* n_pages) {
  if (!p || !n_pages || (cap && !addresses)) return fail(BOOST_EINVAL, "null argument");
  if (p->ctx->device < 0) return fail(BOOST_ENODEV, "plan-only pool");
  if (layer < 0 || static_cast<uint32_t>(layer) >= p->cfg.layers || which < 0 || which > 1)
    return fail(BOOST_EINVAL, "layer %d, tensor %d", layer, which);
  const uint64_t P = p->geom.pages, Hp = p->geom.host_pages, t = 2ull * layer + which;
  *n_pages = P;
  for (uint64_t pg = 0; pg < std::min(P, cap); ++pg)
    addresses[pg] = reinterpret_cast<uint64_t>(
        pg < P - Hp ? p->hbm.base + (t * (P - Hp) + pg) * kPage
                    : p->host[layer].base + (which * Hp + (pg - (P - Hp))) * kPage);
  return BOOST_OK;
}

int boost_kv_block_host_heads(const boost_kv_pool* p, int32_t block, uint32_t* n) {
  if (!p || !n) return fail(BOOST_EINVAL, "null argument");
  if (block < 0 || static_cast<uint32_t>(block) >= p->geom.nb)
    return fail(BOOST_EINVAL, "block %d outside the pool", block);
  *n = p->geom.host_heads[block];
  return BOOST_OK;
}

int boost_kv_alloc(boost_kv_pool* p, uint64_t rid, uint32_t n, int32_t* out) {
  if (!p) return fail(BOOST_EINVAL, "null pool");
  return guarded([&] { return p->dsr.alloc(rid, n, out); });
}

int boost_kv_free(boost_kv_pool* p, uint64_t rid) {
  if (!p) return fail(BOOST_EINVAL, "null pool");
  return guarded([&] { return p->dsr.release(rid); });
}

int boost_kv_fork(boost_kv_pool* p, uint64_t parent, uint64_t child, uint32_t n) {
  if (!p) return fail(BOOST_EINVAL, "null pool");
  return guarded([&] { return p->dsr.fork(parent, child, n); });
}

int boost_kv_unshare(boost_kv_pool* p, uint64_t rid, uint32_t index, int32_t* src, int32_t* dst) {
  if (!p) return fail(BOOST_EINVAL, "null pool");
  return guarded([&] { return p->dsr.unshare(rid, index, src, dst); });
}

int boost_kv_truncate(boost_kv_pool* p, uint64_t rid, uint32_t n_keep) {
  if (!p) return fail(BOOST_EINVAL, "null pool");
  return guarded([&] { return p->dsr.truncate(rid, n_keep); });
}

int boost_kv_compact(boost_kv_pool* p, uint32_t max_moves, int32_t* src, int32_t* dst,
                     uint32_t* n_moves) {
  if (!p) return fail(BOOST_EINVAL, "null pool");
  return guarded([&] { return p->dsr.compact(max_moves, src, dst, n_moves); });
}

int boost_kv_request_blocks(const boost_kv_pool* p, uint64_t rid, int32_t* blocks, uint32_t cap,
                            uint32_t* n) {
  if (!p) return fail(BOOST_EINVAL, "null pool");
  return p->dsr.blocks(rid, blocks, cap, n);
}

int boost_kv_request_type(const boost_kv_pool* p, uint64_t rid, int* type) {
  if (!p) return fail(BOOST_EINVAL, "null pool");
  return p->dsr.type_of(rid, type);
}

int boost_kv_stats(const boost_kv_pool* p, boost_kv_usage* s) {
  if (!p || !s) return fail(BOOST_EINVAL, "null argument");
  s->free_shh = p->dsr.free_shh();
  s->free_local = p->dsr.free_local();
  s->used_blocks = p->dsr.used_blocks();
  s->used_host_head_blocks = p->dsr.used_host_head_blocks();
  s->requests = p->dsr.requests();
  s->shh_requests = p->dsr.shh_requests();
  return BOOST_OK;
}

int boost_kv_write(boost_ctx* ctx, const boost_kv_pool* p, int layer, const int32_t* slots,
                   const void* k, const void* v, int n, void* stream) {
  if (!ctx || !p || !slots || !k || !v) return fail(BOOST_EINVAL, "null argument");
  if (ctx->device < 0 || !p->d_page_table) return fail(BOOST_ENODEV, "plan-only pool");
  if (layer < 0 || static_cast<uint32_t>(layer) >= p->cfg.layers)
    return fail(BOOST_EINVAL, "layer %d", layer);
  if (n < 0) return fail(BOOST_EINVAL, "n=%d", n);
  if (n == 0) return BOOST_OK;
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15)
    return fail(BOOST_EINVAL, "k and v must be 16-byte aligned");
  if (p->format == BOOST_KV_FP4)
    return kv_write4(p, layer, slots, nullptr, 0, nullptr, k, v, n, stream);
  const uint64_t P = p->geom.pages;
  const char* const* pk = p->d_page_table + (2ull * layer) * P;
  const char* const* pv = p->d_page_table + (2ull * layer + 1) * P;
  const int64_t total = static_cast<int64_t>(n) * p->cfg.kv_heads * (p->cfg.head_dim / 8);
  hipLaunchKernelGGL(kv_write_kernel, dim3(static_cast<unsigned>((total + 255) / 256)),
                     dim3(256), 0, static_cast<hipStream_t>(stream), pk, pv, slots,
                     static_cast<const uint4*>(k), static_cast<const uint4*>(v), n,
                     static_cast<int>(p->cfg.kv_heads), static_cast<int>(p->cfg.head_dim),
                     static_cast<int>(p->cfg.block_tokens), static_cast<int>(p->geom.nb));
  BOOST_HIP(hipGetLastError());
  return BOOST_OK;
}

int boost_kv_read(boost_ctx* ctx, const boost_kv_pool* p, int layer, const int32_t* slots, void* k,
                  void* v, int n, void* stream) {
  if (!ctx || !p || !slots || !k || !v) return fail(BOOST_EINVAL, "null argument");
  const char* const *pk, * const *pv;
  if (int rc = kv_layer(p, layer, &pk, &pv)) return rc;
  if (n < 0) return fail(BOOST_EINVAL, "n=%d", n);
  if (n == 0) return BOOST_OK;
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15)
    return fail(BOOST_EINVAL, "k and v must be 16-byte aligned");
  const int H = static_cast<int>(p->cfg.kv_heads), D = static_cast<int>(p->cfg.head_dim);
  const bool fp4 = p->format == BOOST_KV_FP4;
  const int64_t grid = fp4 ? (static_cast<int64_t>(n) + kRows4 - 1) / kRows4 * H
                           : (static_cast<int64_t>(n) * H * (D / 8) + 255) / 256;
  if (grid > 0x7fffffff) return fail(BOOST_EINVAL, "n=%d: grid too large", n);
  const dim3 g(static_cast<unsigned>(grid));
  const auto s = static_cast<hipStream_t>(stream);
  if (fp4)
    hipLaunchKernelGGL(kv_read4_kernel, g, dim3(16 * kRows4), 0, s, pk, pv, slots, static_cast<uint4*>(k),
                       static_cast<uint4*>(v), n, H, static_cast<int>(p->geom.nb));
  else
    hipLaunchKernelGGL(kv_read_kernel, g, dim3(256), 0, s, pk, pv, slots, static_cast<uint4*>(k),
                       static_cast<uint4*>(v), n, H, D, static_cast<int>(p->cfg.block_tokens),
                       static_cast<int>(p->geom.nb));
  BOOST_HIP(hipGetLastError());
  return BOOST_OK;
}

int boost_kv_copy_blocks(boost_ctx* ctx, const boost_kv_pool* p, int layer0, int n_layers,
                         const int32_t* src, const int32_t* dst, int n, void* stream) {
  if (!ctx || !p || (n > 0 && (!src || !dst))) return fail(BOOST_EINVAL, "null argument");
  if (int rc = kv_device(p)) return rc;
  if (layer0 < 0 || n_layers < 1 ||
      static_cast<int64_t>(layer0) + n_layers > static_cast<int64_t>(p->cfg.layers))
    return fail(BOOST_EINVAL, "layers [%d, %d + %d) of %u", layer0, layer0, n_layers,
                p->cfg.layers);
  if (n < 0) return fail(BOOST_EINVAL, "n=%d", n);
  const int nb = static_cast<int>(p->geom.nb), H = static_cast<int>(p->cfg.kv_heads);
  const int tensors = p->d_index ? 3 : 2;
  if (n_layers > 65535 || static_cast<int64_t>(H) * tensors > 65535)
    return fail(BOOST_EINVAL, "grid too large");
  // every destination once, and none of them a source: the order in which
  // the pairs run then makes no difference
  const int rc = guarded([&] {
    std::vector<int32_t> to(dst, dst + n);
    std::sort(to.begin(), to.end());
    for (int i = 0; i < n; ++i) {
      if (src[i] < 0 || src[i] >= nb || dst[i] < 0 || dst[i] >= nb)
        return fail(BOOST_EINVAL, "pair %d: block %d or %d outside the pool", i, src[i], dst[i]);
      if (std::binary_search(to.begin(), to.end(), src[i]))
        return fail(BOOST_EINVAL, "block %d is both read and written", src[i]);
      if (i && to[i] == to[i - 1]) return fail(BOOST_EINVAL, "block %d is written twice", to[i]);
    }
    return BOOST_OK;
  });
  if (rc) return rc;
  const CopyParams P{p->d_page_table, p->geom.pages, p->d_index,
                     static_cast<uint64_t>(p->cfg.layers) * H * nb, layer0, H, nb,
                     H * tensors, p->cfg.block_tokens * p->cfg.head_dim * 2};
  const int rows = p->format == BOOST_KV_FP4 ? (H * tensors + 3) / 4 : H * tensors;
  auto launch = [&](auto per_launch) {
    constexpr int N = decltype(per_launch)::value;
    const auto kernel = p->format == BOOST_KV_FP4 ? copy_blocks_kernel<true, N>
                                                  : copy_blocks_kernel<false, N>;
    for (int i = 0; i < n; i += N) {
      CopyPairs<N> pairs;
      const int m = std::min(n - i, N);
      std::copy_n(src + i, m, pairs.src);
      std::copy_n(dst + i, m, pairs.dst);
      hipLaunchKernelGGL(kernel, dim3(m, rows, n_layers), dim3(256), 0,
                         static_cast<hipStream_t>(stream), P, pairs);
      BOOST_HIP(hipGetLastError());
    }
    return BOOST_OK;
  };
  return n <= kCopyFew ? launch(std::integral_constant<int, kCopyFew>{})
                       : launch(std::integral_constant<int, kCopyPairs>{});
}

}  // extern "C"
