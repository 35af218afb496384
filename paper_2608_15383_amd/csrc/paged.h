// Shared by the kernels over the paged key-value cache (exactmoe_serving.h,
// exactmoe_drafts.h): the cache as they see it, tiles of keys and values for the
// matrix instructions, and the checks of what the calls have in common.
#pragma once

#include <cmath>
#include <type_traits>

#include "device_route.h"
#include "serving.h"

namespace emoe {

// What the kernels need of the cache; strides in bytes.
struct KvView {
  uint8_t *k, *v;
  const float *k_scale, *v_scale;
  int64_t page_bytes;
  int32_t slot_bytes, head_bytes;  // below 2^30, as a page is
  int32_t n_pages, page_log2, n_kv_heads;
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Loads of what is read once: they leave the caches to what is read again.
__device__ __forceinline__ uint4 load_once(const uint4* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// The 16-bit type's matrix instruction (16 x 16 outputs, 32 products each) and
// its pairs of two E4M3 values (exact) of a dword's half.
template <class T>
struct Half16;
template <>
struct Half16<Bf16> {
  __device__ static __forceinline__ f32x4 mfma(uint4 a, uint4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  template <bool kHi>
  __device__ static __forceinline__ uint32_t from_e4m3(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, kHi));
  }
};
template <>
struct Half16<Fp16> {
  __device__ static __forceinline__ f32x4 mfma(uint4 a, uint4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  template <bool kHi>
  __device__ static __forceinline__ uint32_t from_e4m3(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, kHi));
  }
};

constexpr int kTileKeys = 32;   // keys of one wavefront's step

typedef const __attribute__((address_space(4))) int32_t* ConstI32;

// 2^x by the hardware instruction (1 ulp; denormal results are 0).
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// What a part of a softmax with maximum m counts for beside maximum M.  One
// that saw no score counts for 0, by a product: its sums may be NaN.
__device__ __forceinline__ float part_weight(float m, float M) {
  return m == -INFINITY ? 0.f : exp2_hw(m - M);
}

// One tile of 32 keys of one key head, as the matrix instructions take it: two
// halves of two octets, an octet being 8 slots of one page.
//
// Scores: S^T [key][query] = K Q^T.  The A operand's lane (l16, g) holds 8
// dimensions of row l16; any dimensions do, as long as the query's lanes hold
// the same, and any key may be any row.  Row 4r + i of a half is slot
// 2r + (i & 1) of its octet i >> 1.  A load takes one octet, 8 lanes to a slot,
// so that it covers whole 128-byte lines (4 lanes to a slot, the operand's own
// arrangement, read the cache at 5.3 TB/s where this reaches 6): lanes with
// i >> 1 = 0 hold the row's first 4 chunks and the others the next 4, and lanes
// l and l ^ 2 trade what they have of the other one's octet.  All addresses are
// a scalar of the octet plus an offset that a lane keeps.
// Output: O^T [dim][query] = V^T P^T.  The B operand's lane wants 8 keys of
// its query, in any order: those of the rows that its scores are in, so scores
// become weights in the registers that hold them.  The A operand's lane wants
// the same 8 keys of one dimension; it loads kDh / 16 consecutive dimensions of
// each and transposes with byte permutes (32 of them per tile at 128
// dimensions), which keeps values out of LDS.  A query's running maximum, sum
// and output columns all live in lanes l16 = query, so nothing is exchanged
// between queries in the loop.
// Its weights are two 16-bit halves each, what the first one's rounding leaves
// being the second: with them a weight is known to 2^-16 of itself, in bf16
// however small it is, in fp16 only from 2^-9 on.  E4M3 values are exact in bf16
// and take bf16 weights under queries of either type.
template <class T, bool kE4M3, int kDh>
struct Tile {
  typedef Half16<T> H16;
  static constexpr bool kF16Weights = !kE4M3 && T::kType == EMOE_F16;
  typedef typename std::conditional<kF16Weights, Fp16, Bf16>::type W;
  typedef Half16<W> HW;
  static constexpr int kSteps = kDh / 32;
  static constexpr int kItem = kE4M3 ? 1 : 2;
  static constexpr int kChunk = kE4M3 && kDh == 64 ? 8 : 16;  // bytes of a lane's load
  static constexpr int kChunkWords = kChunk / 4;
  static constexpr int kChunkDims = kChunk / kItem;
  static constexpr int kSub = kChunkDims / 8;              // steps of a chunk
  static constexpr int kPairs = kDh / (8 * kChunkDims);    // loads of an octet
  static constexpr int kDims = kDh / 16;                   // output dimensions of a lane
  static constexpr int kVWords = kDims * kItem / 4;
  static constexpr bool kSplitV = !kE4M3 && kDh == 256;    // two 16-byte loads, 256 bytes apart

  uint32_t k[4][kPairs][kChunkWords];
  uint32_t v[8][kVWords];

  // The first of the 8 dimensions that lane group g holds in step c.
  __device__ static __forceinline__ int q_dim(int c, int g) {
    return kChunkDims * (4 * (c / kSub) + g) + 8 * (c % kSub);
  }
  // Output dimension of matrix row m of accumulator c.
  __device__ static __forceinline__ int out_dim(int m, int c) {
    return kSplitV ? 128 * (c >> 3) + 8 * m + (c & 7) : kDims * m + c;
  }
  // A lane's offset from an octet's first slot: its key's chunk, its value's
  // dimensions (of the slot 2g; the slot after it for odd i).
  __device__ static __forceinline__ uint32_t k_offset(int lane, int slot_bytes) {
    const int m = lane & 15, slot = 2 * (m >> 2) + (m & 1);
    return slot * slot_bytes + kChunk * (2 * (m & 2) + (lane >> 4));
  }
  __device__ static __forceinline__ uint32_t v_offset(int lane, int slot_bytes) {
    return 2 * (lane >> 4) * slot_bytes + (kSplitV ? 16 : kVWords * 4) * (lane & 15);
  }

  __device__ __forceinline__ void load_k(const uint8_t* const (&octet)[4], uint32_t off) {
#pragma unroll
    for (int o = 0; o < 4; ++o)
#pragma unroll
      for (int p = 0; p < kPairs; ++p) {
        const uint8_t* at = octet[o] + off + 8 * kChunk * p;
        if constexpr (kChunkWords == 4) {
          const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at));
          k[o][p][0] = w.x, k[o][p][1] = w.y, k[o][p][2] = w.z, k[o][p][3] = w.w;
        } else {
          const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(at));
          k[o][p][0] = w.x, k[o][p][1] = w.y;
        }
      }
  }
  __device__ __forceinline__ void load_v(const uint8_t* const (&octet)[4], int slot_bytes,
                                         uint32_t off) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint8_t* p = octet[j >> 1] + (j & 1) * slot_bytes + off;
      if constexpr (kVWords == 1) {
        v[j][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
      } else if constexpr (kVWords == 2) {
        const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
        v[j][0] = w.x, v[j][1] = w.y;
      } else {
#pragma unroll
        for (int u = 0; u < kVWords / 4; ++u) {
          const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 256 * u));
          v[j][4 * u] = w.x, v[j][4 * u + 1] = w.y, v[j][4 * u + 2] = w.z, v[j][4 * u + 3] = w.w;
        }
      }
    }
  }
  // Scores of the half h's rows: step by step, chunks of the first octet and
  // of the second traded between lanes l and l ^ 2.
  __device__ __forceinline__ void scores(const uint4 (&q)[kSteps], bool second, f32x4 (&s)[2]) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < kPairs; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t c0[kChunkWords], c1[kChunkWords];
#pragma unroll
        for (int w = 0; w < kChunkWords; ++w) {
          const uint32_t a = k[2 * h][p][w], b = k[2 * h + 1][p][w];
          const uint32_t a2 = __builtin_amdgcn_update_dpp(0, (int)a, 0x4E, 0xF, 0xF, true);
          const uint32_t b2 = __builtin_amdgcn_update_dpp(0, (int)b, 0x4E, 0xF, 0xF, true);
          c0[w] = second ? b2 : a;
          c1[w] = second ? b : a2;
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int sub = 0; sub < kSub; ++sub) {
            const uint32_t(&c)[kChunkWords] = half ? c1 : c0;
            uint4 x;
            if constexpr (kE4M3) {
              const uint32_t lo = c[2 * sub], hi = c[2 * sub + 1];
              x = make_uint4(H16::template from_e4m3<false>(lo), H16::template from_e4m3<true>(lo),
                             H16::template from_e4m3<false>(hi), H16::template from_e4m3<true>(hi));
            } else {
              x = make_uint4(c[0], c[1], c[2], c[3]);
            }
            s[h] = H16::mfma(x, q[(2 * p + half) * kSub + sub], s[h]);
          }
      }
  }
  // Values of keys that are not there become 0: a weight of 0 does not undo a NaN.
  __device__ __forceinline__ void clear_v(uint32_t there) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int w = 0; w < kVWords; ++w) v[j][w] = (there >> j) & 1 ? v[j][w] : 0u;
  }
  // Lets the compiler know nothing of the values any more: a further add_pair would
  // have it keep all transposed pairs, in 45 registers more.
  __device__ __forceinline__ void transpose_again() {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int w = 0; w < kVWords; ++w) asm volatile("" : "+v"(v[j][w]));
  }
  // The pair of dimensions (2w, 2w + 1) of key j.
  template <int kW>
  __device__ __forceinline__ uint32_t pair(int j) const {
    if constexpr (kE4M3) return HW::template from_e4m3<(kW & 1) != 0>(v[j][kW >> 1]);
    else return v[j][kW];
  }
  template <int kW>
  __device__ __forceinline__ void add_pair(uint4 hi, uint4 lo, f32x4 (&acc)[kDims]) const {
    uint32_t e[4], o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = pair<kW>(2 * i), b = pair<kW>(2 * i + 1);
      e[i] = __builtin_amdgcn_perm(b, a, 0x05040100u);
      o[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    }
    const uint4 ve = make_uint4(e[0], e[1], e[2], e[3]), vo = make_uint4(o[0], o[1], o[2], o[3]);
    acc[2 * kW] = HW::mfma(ve, hi, acc[2 * kW]);
    acc[2 * kW + 1] = HW::mfma(vo, hi, acc[2 * kW + 1]);
    acc[2 * kW] = HW::mfma(ve, lo, acc[2 * kW]);
    acc[2 * kW + 1] = HW::mfma(vo, lo, acc[2 * kW + 1]);
    if constexpr (kW + 1 < kDims / 2) add_pair<kW + 1>(hi, lo, acc);
  }
};

// The pages of a tile's four octets of keys (a page has 8 slots or more).
struct Octets {
  int32_t page[4];
};
__device__ __forceinline__ Octets octets_of(const KvView& kv, ConstI32 table, int key0, int n) {
  Octets o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = key0 + 8 * i;
    o.page[i] = j < n ? table[j >> kv.page_log2] : -1;
  }
  return o;
}

// Inclusive sum over the wavefront by DPP moves (8 cycles each; a shuffle
// through LDS takes a hundred).
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31
  return v;
}

// ---------------------------------------------------------------- the host's side: checks
inline int32_t check_kv(const emoe_paged_kv* kv) {
  if (!kv) return report_error(EMOE_EINVAL, "kv is NULL");
  if (!kv->k_pages || !kv->v_pages) return report_error(EMOE_EINVAL, "NULL pages");
  if (kv->dtype != EMOE_BF16 && kv->dtype != EMOE_F16 && kv->dtype != EMOE_E4M3)
    return report_error(EMOE_EINVAL, "cache type %d: need bf16, fp16 or e4m3", kv->dtype);
  if (kv->dtype != EMOE_E4M3 && (kv->k_scale || kv->v_scale))
    return report_error(EMOE_EINVAL, "scales with a 16-bit cache");
  if (!kv->k_scale != !kv->v_scale) return report_error(EMOE_EINVAL, "one of k_scale and v_scale is NULL");
  const int ps = kv->page_size, dh = kv->head_dim;
  if (ps < 8 || ps > 1024 || (ps & (ps - 1)))
    return report_error(EMOE_ESHAPE, "page_size %d: need a power of two from 8 to 1024", ps);
  if (dh != 64 && dh != 128 && dh != 256)
    return report_error(EMOE_ESHAPE, "head_dim %d: need 64, 128 or 256", dh);
  if (kv->n_pages < 1 || kv->n_kv_heads < 1)
    return report_error(EMOE_ESHAPE, "need n_pages and n_kv_heads >= 1 (got %d, %d)", kv->n_pages,
                        kv->n_kv_heads);
  const int64_t item = kv->dtype == EMOE_E4M3 ? 1 : 2, unit = 16 / item;
  const int64_t hk = kv->n_kv_heads, most = (int64_t)1 << 30;
  const int64_t ss = kv->slot_stride, hs = hk == 1 ? dh : kv->head_stride;
  const int64_t pg = kv->n_pages == 1 ? INT64_MAX : kv->page_stride;
  if (ss % unit || hs % unit || (pg != INT64_MAX && pg % unit) || !aligned16(kv->k_pages) || !aligned16(kv->v_pages))
    return report_error(EMOE_EINVAL, "pages and strides must be multiples of 16 bytes");
  // Bounded before they are multiplied.
  if (ss < dh || hs < dh || ss > most || hs > most || hk > most || hk * hs > most || ps * ss > most)
    return report_error(EMOE_ESHAPE, "slot_stride %lld or head_stride %lld: below head_dim, or a page "
                        "above 2^30 bytes", (long long)ss, (long long)hs);
  const bool heads_inside = ss >= (hk - 1) * hs + dh && pg >= (ps - 1) * ss + (hk - 1) * hs + dh;
  const bool slots_inside = hs >= (ps - 1) * ss + dh && pg >= (hk - 1) * hs + (ps - 1) * ss + dh;
  if (!heads_inside && !slots_inside)
    return report_error(EMOE_ESHAPE, "page, slot and head strides %lld, %lld, %lld overlap",
                        (long long)kv->page_stride, (long long)ss, (long long)hs);
  if (((ps - 1) * ss + (hk - 1) * hs + dh) * item > most)
    return report_error(EMOE_ESHAPE, "a page above 2^30 bytes");
  return EMOE_OK;
}

inline KvView view_of(const emoe_paged_kv& kv) {
  const int64_t item = kv.dtype == EMOE_E4M3 ? 1 : 2;
  KvView w;
  w.k = static_cast<uint8_t*>(kv.k_pages);
  w.v = static_cast<uint8_t*>(kv.v_pages);
  w.k_scale = kv.k_scale;
  w.v_scale = kv.v_scale;
  w.page_bytes = kv.n_pages == 1 ? 0 : kv.page_stride * item;
  w.slot_bytes = (int32_t)(kv.slot_stride * item);
  w.head_bytes = kv.n_kv_heads == 1 ? 0 : (int32_t)(kv.head_stride * item);
  w.n_pages = kv.n_pages;
  w.page_log2 = __builtin_ctz((unsigned)kv.page_size);
  w.n_kv_heads = kv.n_kv_heads;
  return w;
}

// Shared by both calls: the 16-bit side and the page table.
inline int32_t check_io(const emoe_paged_kv& kv, int32_t dtype, const int32_t* table, int32_t n_seqs,
                 int32_t table_width, int64_t table_stride) {
  if (dtype != EMOE_BF16 && dtype != EMOE_F16)
    return report_error(EMOE_EINVAL, "type %d: need bf16 or fp16", dtype);
  if (kv.dtype != EMOE_E4M3 && kv.dtype != dtype)
    return report_error(EMOE_EINVAL, "type %d over a 16-bit cache of type %d", dtype, kv.dtype);
  if (n_seqs < 0 || table_width < 0) return report_error(EMOE_EINVAL, "negative n_seqs or table_width");
  if (n_seqs > 0 && table_width > 0 && !table) return report_error(EMOE_EINVAL, "page_table is NULL");
  if (n_seqs > 1 && table_stride < table_width)
    return report_error(EMOE_EINVAL, "table_stride %lld below table_width %d", (long long)table_stride,
                        table_width);
  return EMOE_OK;
}

inline int32_t check_rows(const char* what, const void* p, int64_t stride, int64_t rows, int64_t width) {
  if (!p) return report_error(EMOE_EINVAL, "%s is NULL", what);
  if (!aligned16(p) || (rows > 1 && stride % 8))
    return report_error(EMOE_EINVAL, "%s: need 16-byte aligned rows", what);
  if (rows > 1 && stride < width)
    return report_error(EMOE_EINVAL, "%s: row stride %lld below the row's %lld elements", what,
                        (long long)stride, (long long)width);
  return EMOE_OK;
}

inline int32_t launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return report_error(EMOE_EHIP, "%s launch: %s", what, hipGetErrorString(e));
  return EMOE_OK;
}

// Bounds of the calls' integers: keys of a row and what a tile adds to them stay
// within 32 bits, and lines times threads within a grid; an appended token's
// items (at most 2^24 of q and, as a page's slots are below 2^30 elements, 2^27 of
// k and v) and what a step of its workgroups adds to them stay within 32 bits.
constexpr int32_t kMostKeys = 1 << 30, kMostHeads = 1 << 20;

}  // namespace emoe
