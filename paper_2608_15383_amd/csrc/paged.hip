// The paged key-value cache (exactmoe_serving.h): append with the rotary
// positions on the way, and the attention of one new token per row.
#include <cmath>
#include <type_traits>

#include "device_rope.h"
#include "device_route.h"
#include "serving.h"

using namespace emoe;

namespace {

constexpr int kThreads = 256;

// What the kernels need of the cache; strides in bytes.
struct KvView {
  uint8_t *k, *v;
  const float *k_scale, *v_scale;
  int64_t page_bytes;
  int32_t slot_bytes, head_bytes;  // below 2^30, as a page is
  int32_t n_pages, page_log2, n_kv_heads;
};

// ---------------------------------------------------------------- append
struct AppendArg {
  KvView kv;
  const uint16_t *q, *k, *v;
  uint16_t* q_out;
  const int32_t *positions, *seqs, *table;
  const double* inv_freq;
  int64_t q_stride, k_stride, v_stride, qo_stride, table_stride;
  int64_t token0;
  int32_t n_heads, n_seqs, table_width, rotary_dim;
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Loads of what is read once: they leave the caches to what is read again.
__device__ __forceinline__ uint4 load_once(const uint4* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
}

// A workgroup takes one token: its angles' cosines and sines once (fp64, shared
// by all heads), then items of two 16-byte chunks (16 dimensions) of one head of
// q, k or v: a chunk of the first half of the rotated dimensions and the one it
// turns with, or, interleaved or not rotated, two neighbours.  blockIdx.y
// splits the items of small calls.  Bound by HBM: every value is read and
// written once; 7,919 tokens of 32 + 16 heads of 128 take 38.8 us, 5.0 TB/s,
// what a plain copy reaches.  Two tokens to a workgroup 41.9 us, four 44.6,
// eight 44.4; without the streaming loads 39.5; with streaming stores 49.2.
template <class T, bool kE4M3, bool kInter, int kDh>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(AppendArg a) {
  __shared__ float2 cs[kDh / 2];
  constexpr int kPieces = kDh / 16;
  const int64_t t = a.token0 + blockIdx.x;
  const int p = a.positions[t], s = a.seqs ? a.seqs[t] : (int)t;
  if (p < 0 || (uint32_t)s >= (uint32_t)a.n_seqs) return;
  int64_t slot_at = -1;  // byte offset of the token's slot, -1: none
  const int col = p >> a.kv.page_log2;
  if (col < a.table_width) {
    const int page = a.table[(int64_t)s * a.table_stride + col];
    if ((uint32_t)page < (uint32_t)a.kv.n_pages)
      slot_at = page * a.kv.page_bytes +
                (int64_t)(p & ((1 << a.kv.page_log2) - 1)) * a.kv.slot_bytes;
  }
  for (int i = threadIdx.x; i < a.rotary_dim / 2; i += kThreads) {
    float2 w;
    rope_cos_sin((double)p * a.inv_freq[i], w.x, w.y);
    cs[i] = w;
  }
  __syncthreads();
  const int q_heads = a.q ? a.n_heads : 0;
  const int n_items = (q_heads + 2 * a.kv.n_kv_heads) * kPieces;
  for (int j = blockIdx.y * kThreads + threadIdx.x; j < n_items; j += gridDim.y * kThreads) {
    int h = j / kPieces;
    const int pc = j % kPieces;
    const int kind = h < q_heads ? 0 : (h < q_heads + a.kv.n_kv_heads ? 1 : 2);
    h -= kind == 0 ? 0 : (kind == 1 ? q_heads : q_heads + a.kv.n_kv_heads);
    if (kind != 0 && slot_at < 0) continue;
    // The two chunks (8 dimensions each).
    const bool turns = kind != 2 && 16 * pc < a.rotary_dim;
    int c0 = 2 * pc, c1 = 2 * pc + 1;
    if (!kInter && turns) {
      c0 = pc;
      c1 = pc + a.rotary_dim / 16;
    }
    const uint16_t* src = kind == 0   ? a.q + t * a.q_stride
                          : kind == 1 ? a.k + t * a.k_stride
                                      : a.v + t * a.v_stride;
    const uint4* row = reinterpret_cast<const uint4*>(src + (int64_t)h * kDh);
    float x0[8], x1[8];
    up8<T>(load_once(row + c0), x0);
    up8<T>(load_once(row + c1), x1);
    if (turns) {
      if constexpr (kInter) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 w0 = cs[8 * pc + i], w1 = cs[8 * pc + 4 + i];
          const float a0 = x0[2 * i], b0 = x0[2 * i + 1], a1 = x1[2 * i], b1 = x1[2 * i + 1];
          x0[2 * i] = fmaf(a0, w0.x, -(b0 * w0.y));
          x0[2 * i + 1] = fmaf(a0, w0.y, b0 * w0.x);
          x1[2 * i] = fmaf(a1, w1.x, -(b1 * w1.y));
          x1[2 * i + 1] = fmaf(a1, w1.y, b1 * w1.x);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 w = cs[8 * pc + i];
          const float a0 = x0[i], b0 = x1[i];
          x0[i] = fmaf(a0, w.x, -(b0 * w.y));
          x1[i] = fmaf(a0, w.y, b0 * w.x);
        }
      }
    }
    if (kind == 0) {
      uint4* dst = reinterpret_cast<uint4*>(a.q_out + t * a.qo_stride + (int64_t)h * kDh);
      dst[c0] = down8<T>(x0);
      dst[c1] = down8<T>(x1);
    } else {
      uint8_t* dst = (kind == 1 ? a.kv.k : a.kv.v) + slot_at + (int64_t)h * a.kv.head_bytes;
      if constexpr (kE4M3) {
        const float* scale = kind == 1 ? a.kv.k_scale : a.kv.v_scale;
        if (scale) {
          const float s = scale[h];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x0[i] /= s;
            x1[i] /= s;
          }
        }
        reinterpret_cast<uint2*>(dst)[c0] = down8_e4m3(x0);
        reinterpret_cast<uint2*>(dst)[c1] = down8_e4m3(x1);
      } else {
        reinterpret_cast<uint4*>(dst)[c0] = down8<T>(x0);
        reinterpret_cast<uint4*>(dst)[c1] = down8<T>(x1);
      }
    }
  }
}

// ---------------------------------------------------------------- attention
struct AttendArg {
  KvView kv;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  const int32_t *lengths, *seqs, *table;
  uint32_t* tickets;
  float* parts;
  int64_t q_stride, out_stride, table_stride;
  float scale;
  int32_t row0, rows, n_heads, group, q_tiles, n_seqs, table_width, max_keys, window;
  int32_t workers, part_floats;
};

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
constexpr int kMaxRows = 1024;  // rows of one launch

typedef const __attribute__((address_space(4))) int32_t* ConstI32;

// 2^x by the hardware instruction (1 ulp; denormal results are 0).
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// What a part of a softmax with maximum m counts for beside maximum M.  One
// that saw no score counts for 0, by a product: its sums may be NaN.
__device__ __forceinline__ float part_weight(float m, float M) {
  return m == -INFINITY ? 0.f : exp2_hw(m - M);
}

// The keys that row `row` of the call sees: [first, n).
struct Span {
  int first, n, seq;
};
__device__ __forceinline__ Span span_of(const AttendArg& a, int row) {
  Span s;
  s.seq = a.seqs ? a.seqs[row] : row;
  int n = 0;
  if ((uint32_t)s.seq < (uint32_t)a.n_seqs) {
    n = max(0, min(a.lengths[row], a.max_keys));
    n = (int)min((int64_t)n, (int64_t)a.table_width << a.kv.page_log2);
  }
  s.n = n;
  s.first = a.window > 0 ? max(0, n - a.window) : 0;
  return s;
}
// Its units, of a tile for each of kWaves wavefronts, from the tile of its first
// key on; a row without keys has one, which writes its zeros.
template <int kWaves>
__device__ __forceinline__ int units_of(int first, int n) {
  const int t0 = first / kTileKeys, t1 = (n + kTileKeys - 1) / kTileKeys;
  return max(1, (t1 - t0 + kWaves - 1) / kWaves);
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
__device__ __forceinline__ Octets octets_of(const AttendArg& a, ConstI32 table, int key0, int n) {
  Octets o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = key0 + 8 * i;
    o.page[i] = j < n ? table[j >> a.kv.page_log2] : -1;
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

// How the rows of a launch are cut for the workers (workgroups) of a line: rows
// stand behind each other, each in a number of slots, and a worker takes `run`
// slots.  Either slots are units and every worker takes the same number of them,
// wherever rows begin and end: best where a worker has many.  Or a row has at
// most ceil(units / target) slots and every worker one, so that its run never
// spans two rows, which costs a run about four units more.
// To join a shared row costs 3 to 8 us, a unit of a worker's own about 1.4 us per
// 64 KB (what a CU keeps in flight; smaller units 1 us): rows stay whole unless
// the longest gives up pays_units or more.  Whole against cut, 8 key heads, 16
// bits: 4 rows of 1,024 keys of 128 dimensions 19.0 and 11.1 us, 16 of 512 13.4
// and 15.3, 4 of 1,024 of 64 dimensions 14.0 and 9.7; 4 key heads of 256
// dimensions, 16 rows of 512 17.8 and 14.2, of 2,048 54.0 and 28.4.  A target of
// more than slack_units above the equal runs' gives way to those: 32 rows of up to
// 2,000 keys, eight wavefronts, 31.4 us with a slack of 6 and 27.0 with 1.
constexpr int slack_units(int waves) { return waves == 8 ? 1 : 6; }
constexpr int pays_units(int unit_bytes) { return unit_bytes > 65536 ? 2 : 4; }
__device__ __forceinline__ int slot_units(int units, int target) {
  if (target == 0) return 1;
  const uint32_t parts = (uint32_t)(units + target - 1) / (uint32_t)target;
  return (int)((uint32_t)(units + parts - 1) / parts);
}
__device__ __forceinline__ int slots_of(int units, int target) {
  if (target == 0 || units == 0) return units;
  const int each = slot_units(units, target);
  return (int)((uint32_t)(units + each - 1) / (uint32_t)each);
}

// Split over the caches' lengths, as above; a worker's kWaves wavefronts take
// every kWaves-th tile of its units.  Outputs that it covers whole it writes; of
// the others (at most its first and its last) it leaves maximum, sum and unscaled
// output in the workspace, and the last of such an output's workers to finish
// joins them in the rows' order (nobody waits).  Key heads (times tiles of 16
// query heads) are the lines: workgroups next to each other take the same keys of
// different heads, which lie next to each other in memory.
// Bound by HBM where there are keys enough: per tile and wavefront 16 KB (16
// bits, 128 dimensions) against about 250 vector and 24 matrix instructions.
// 131,072 keys of 8 heads of 128 take 91.5 us, 5.9 TB/s, of the 6.5 that this
// pattern of reads reaches without any arithmetic; 128 rows over 8 bits 279 us,
// 5.3 TB/s of 6.0 (ragged rows; heads of one 128-byte line each).  Short calls
// are bound by the chain of trips to memory (lengths, page table, keys, parts,
// ticket, parts again): 302 keys take 8.2 us.
template <class T, bool kE4M3, int kDh, int kWaves>
__global__ __launch_bounds__(64 * kWaves, kDh == 256 ? 1 : 2) void paged_attention_kernel(AttendArg a) {
  constexpr int kThreads = 64 * kWaves;
  typedef Tile<T, kE4M3, kDh> Tl;
  constexpr int kPays = pays_units(kWaves * kTileKeys * 2 * kDh * Tl::kItem);
  // fp16 weights begin at 2^7: there is room above, but little below.
  constexpr float kLead = Tl::kF16Weights ? 7.f : 0.f;
  constexpr int kRow = kDh + 4;  // padded: lanes 16 apart in dimensions, 1 in queries
  constexpr bool kWhole = kWaves == 1;  // a row to a workgroup, nothing shared
  constexpr int kRows = kWhole ? 1 : kMaxRows, kJoiners = kWhole ? 1 : kThreads;
  __shared__ int pre[kRows + 1], len[kRows], seq[kRows];
  __shared__ int wave_sum[kWaves], wave_most[kWaves];
  __shared__ float ms[kWaves][16], ls[kWaves][16];
  __shared__ __attribute__((aligned(16))) float os[kWaves][16][kRow];
  __shared__ float4 striped[kJoiners];
  __shared__ float striped_m[kJoiners], striped_l[kJoiners];
  __shared__ int last[2], first_row;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const uint32_t k_off = Tl::k_offset(lane, a.kv.slot_bytes);
  const uint32_t v_off = Tl::v_offset(lane, a.kv.slot_bytes);

  // Workgroups of one key head's tiles of queries are 8 apart, on one die, so that
  // its L2 serves what the second reads again (21 rows of up to 11,854 keys, 24
  // queries to a key head: 40.5 -> 33 us).
  const int chunk = blockIdx.x / (8 * a.q_tiles), at = blockIdx.x % (8 * a.q_tiles);
  const int pairs = min(8, a.workers * a.kv.n_kv_heads - 8 * chunk);
  const int pair = 8 * chunk + at % pairs, qt = at / pairs;
  const int w = pair / a.kv.n_kv_heads, hk = pair % a.kv.n_kv_heads;
  const int Y = a.kv.n_kv_heads * a.q_tiles, y = hk * a.q_tiles + qt;
  const bool few = a.rows <= 64;
  int n_lane = 0, seq_lane = 0, before_lane = 0, slots_lane = 1;
  int run = 1, target = kWhole ? INT32_MAX / 2 : 0, u = 0, u_end = 1, row = kWhole ? w : 0;
  if constexpr (!kWhole) {
    // How the rows are cut, and where this worker's run of slots begins.  Up to
    // 64 rows every wavefront finds out by itself, a row per lane, and keeps them
    // in its lanes; more rows take the workgroup and LDS.
    const int per = few ? 1 : (a.rows + kThreads - 1) / kThreads, r0 = few ? lane : tid * per;
    constexpr int kPer = kMaxRows / kThreads;
    int units_[kPer], total = 0, most = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      units_[i] = 0;
      if (i < per && r0 + i < a.rows) {
        const Span s = span_of(a, a.row0 + r0 + i);
        if (few) {
          n_lane = s.n;
          seq_lane = s.seq;
        } else {
          len[r0 + i] = s.n;
          seq[r0 + i] = s.seq;
        }
        units_[i] = units_of<kWaves>(s.first, s.n);
      }
      total += units_[i];
      most = max(most, units_[i]);
    }
    // Sums over the rows; `before` is what the rows before this thread's have.
    auto sum_rows = [&](int v, int& before) -> int {
      const int incl = wave_scan(v);
      before = incl - v;
      const int all = __builtin_amdgcn_readlane(incl, 63);
      if (few) return all;
      __syncthreads();
      if (lane == 0) wave_sum[wave] = all;
      __syncthreads();
      int sum = 0;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        before += i < wave ? wave_sum[i] : 0;
        sum += wave_sum[i];
      }
      return __builtin_amdgcn_readfirstlane(sum);
    };
    int before;
    total = sum_rows(total, before);
    most = (int)wave_reduce_u32<true>((uint32_t)most);
    if (!few) {
      if (lane == 0) wave_most[wave] = most;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kWaves; ++i) most = max(most, wave_most[i]);
    }
    most = __builtin_amdgcn_readfirstlane(most);
    int all = total;
    run = (total + a.workers - 1) / a.workers;
    if (a.rows <= a.workers) {
      // The smallest target tried for which the workers suffice; they do for the
      // last one, since the sum of ceil(units / target) <= total / target + rows.
      const int spare = a.workers - a.rows, enough = spare ? min(most, (total + spare - 1) / spare) : most;
      int t = most - run < kPays ? most : run;
      while (true) {
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) mine += i < per ? slots_of(units_[i], t) : 0;
        const int sum = sum_rows(mine, before);
        if (t < most && t > run + slack_units(kWaves)) break;  // equal runs, then
        if (sum <= a.workers || t >= enough) {
          target = t;
          all = sum;
          run = (sum + a.workers - 1) / a.workers;
          break;
        }
        t = min(t + max(1, t / 4), max(enough, t + 1));
      }
    }
    if (target == 0) {
      int mine = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) mine += units_[i];
      all = sum_rows(mine, before);
    }
    if ((int64_t)w * run >= all) return;  // the same for the whole workgroup
    u_end = min((w + 1) * run, all);
    u = w * run;
    before_lane = before;
    slots_lane = slots_of(units_[0], target);
    if (few) {
      row = (int)__builtin_ctzll(__ballot(u >= before && u < before + slots_lane));
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (i < per && r0 + i < a.rows) {
          const int n = slots_of(units_[i], target);
          pre[r0 + i] = before;
          if (u >= before && u < before + n) first_row = r0 + i;
          before += n;
        }
      }
      if (tid == 0) pre[a.rows] = all;
      __syncthreads();
      row = first_row;
    }
  }
  // A row's first slot and slots.
  auto slots_at = [&](int r, int& base) -> int {
    if constexpr (kWhole) {
      base = 0;
      return 1;
    }
    if (few) {
      base = __builtin_amdgcn_readlane(before_lane, r);
      return __builtin_amdgcn_readlane(slots_lane, r);
    }
    base = __builtin_amdgcn_readfirstlane(pre[r]);
    return __builtin_amdgcn_readfirstlane(pre[r + 1]) - base;
  };
  bool first_segment = true;
  int waiting = 0, shared0 = 0, shared1 = 0;  // this run's outputs that other workers share
  const int head0 = hk * a.group + qt * 16;
  const int heads = min(16, a.group - qt * 16);
  float scale = a.scale * 1.4426950408889634f;
  if (kE4M3 && a.kv.k_scale) scale *= a.kv.k_scale[hk];
  const float vs = kE4M3 && a.kv.v_scale ? a.kv.v_scale[hk] : 1.f;
  auto store_out = [&](int64_t grow, int h, int d, float4 o, float M, float L) {
    const float inv = L == 0.f ? 0.f : vs / L;
    uint2 r;
    r.x = T::down(o.x * inv) | (T::down(o.y * inv) << 16);
    r.y = T::down(o.z * inv) | (T::down(o.w * inv) << 16);
    *reinterpret_cast<uint2*>(a.out + grow * a.out_stride + (int64_t)(head0 + h) * kDh + d) = r;
    if (d == 0 && a.lse)
      a.lse[grow * a.n_heads + head0 + h] =
          L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
  };
  for (; u < u_end; ++row) {
    row = __builtin_amdgcn_readfirstlane(row);
    int base;
    const int row_slots = slots_at(row, base);
    int n, sq;
    if constexpr (kWhole) {
      const Span s = span_of(a, a.row0 + row);
      n = __builtin_amdgcn_readfirstlane(s.n);
      sq = __builtin_amdgcn_readfirstlane(s.seq);
    } else {
      n = few ? __builtin_amdgcn_readlane(n_lane, row) : __builtin_amdgcn_readfirstlane(len[row]);
      sq = few ? __builtin_amdgcn_readlane(seq_lane, row) : __builtin_amdgcn_readfirstlane(seq[row]);
    }
    const int first = a.window > 0 ? max(0, n - a.window) : 0;
    const int units = units_of<kWaves>(first, n), each = slot_units(units, target);
    const int s0 = u - base, s1 = min(row_slots, s0 + (u_end - u));
    const int c0 = s0 * each, c1 = min(units, s1 * each);
    const int64_t grow = a.row0 + row;

    uint4 q[Tl::kSteps];
#pragma unroll
    for (int c = 0; c < Tl::kSteps; ++c) {
      q[c] = make_uint4(0, 0, 0, 0);
      if (l16 < heads)
        q[c] = *reinterpret_cast<const uint4*>(a.q + grow * a.q_stride +
                                               (int64_t)(head0 + l16) * kDh + Tl::q_dim(c, g));
    }
    f32x4 acc[Tl::kDims];
#pragma unroll
    for (int c = 0; c < Tl::kDims; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    const int t0 = first / kTileKeys;
    const int t_end = min(t0 + c1 * kWaves, (n + kTileKeys - 1) / kTileKeys);
    int t = t0 + c0 * kWaves + wave;
    const ConstI32 table = (ConstI32)(a.table + (int64_t)sq * a.table_stride);
    const uint8_t* kbase = a.kv.k + (int64_t)hk * a.kv.head_bytes;
    const uint8_t* vbase = a.kv.v + (int64_t)hk * a.kv.head_bytes;
    const int slot_mask = (1 << a.kv.page_log2) - 1;

    // The tile's octets (of page 0 where there is no page: any place that may
    // be read), from the first byte of their slots.
    auto place = [&](const Octets& o, int key0, int64_t (&off)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int page = (uint32_t)o.page[i] < (uint32_t)a.kv.n_pages ? o.page[i] : 0;
        off[i] = page * a.kv.page_bytes + (int64_t)((key0 + 8 * i) & slot_mask) * a.kv.slot_bytes;
      }
    };
    Tl tile;
    auto load_k = [&](const int64_t (&off)[4]) {
      const uint8_t* const at[4] = {kbase + off[0], kbase + off[1], kbase + off[2], kbase + off[3]};
      tile.load_k(at, k_off);
    };
    auto load_v = [&](const int64_t (&off)[4]) {
      const uint8_t* const at[4] = {vbase + off[0], vbase + off[1], vbase + off[2], vbase + off[3]};
      tile.load_v(at, a.kv.slot_bytes, v_off);
    };

    Octets now, next;
    int64_t off[4];
    if (t < t_end) {
      now = octets_of(a, table, t * kTileKeys, n);
      place(now, t * kTileKeys, off);
      load_k(off);
      load_v(off);
      if (t + kWaves < t_end) next = octets_of(a, table, (t + kWaves) * kTileKeys, n);
    }
    while (t < t_end) {
      const int key0 = t * kTileKeys, tn = t + kWaves;
      const bool more = tn < t_end;
      f32x4 s[2];
      tile.scores(q, (lane & 2) != 0, s);
      if (more) {
        place(next, tn * kTileKeys, off);
        load_k(off);
      }
      float z[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = s[j >> 2][j & 3] * scale;
      bool whole = key0 >= first && key0 + kTileKeys <= n;
#pragma unroll
      for (int i = 0; i < 4; ++i) whole = whole && (uint32_t)now.page[i] < (uint32_t)a.kv.n_pages;
      if (!whole) {
        uint32_t there = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int key = key0 + 8 * (j >> 1) + 2 * g + (j & 1);
          if (key >= first && key < n && (uint32_t)now.page[j >> 1] < (uint32_t)a.kv.n_pages)
            there |= 1u << j;
          else z[j] = -INFINITY;
        }
        tile.clear_v(there);
      }
      // The exponent that the weights refer to follows the maximum only when a
      // score exceeds it by 8: until then they stay below 2^(8 + kLead), and
      // nothing is rescaled.
      float top = z[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) top = fmaxf(top, z[j]);
      if (__any(top > m + (8.f + kLead))) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m2 = fmaxf(m, top - kLead);
        const float shrink = m2 == -INFINITY ? 0.f : exp2_hw(m - m2);
        m = m2;
        l *= shrink;
#pragma unroll
        for (int c = 0; c < Tl::kDims; ++c) acc[c] *= shrink;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      float p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        p[j] = exp2_hw(z[j] - ref);
        l += p[j];
      }
      // fp16 weights below 2^-9 (a key that draws most of the weight to itself
      // leaves all others there) are added in turns of their own, 2^24 and 2^48
      // times as large, to sums as much larger; the products by powers of two are
      // exact.  Weights below 2^-57, 2^-64 of the largest, would not show: 2^20 of
      // them times the largest value are 2^-28, below fp16's smallest half.  To look
      // for small weights costs 1% to 6% (131,072 keys 91.3 -> 91.9 us, 300 rows of
      // up to 60 keys 10.6 -> 11.3), a turn more 0.5% to 20% (one key 25 nats above
      // all others: 131,072 keys 91.7 -> 92.1, 302 keys 8.1 -> 9.8).
      float lift = 1.f;
      while (true) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = p[j];
        bool rest = false;
        if constexpr (Tl::kF16Weights) {
          uint32_t least = ~0u;  // the bits, less 1, of the smallest weight above 0
#pragma unroll
          for (int j = 0; j < 8; ++j) least = min(least, __float_as_uint(p[j]) - 1u);
          rest = __any(least < __float_as_uint(0x1p-9f) - 1u);
          if (rest) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const bool small = p[j] < 0x1p-9f;
              y[j] = small ? 0.f : p[j];
              p[j] = small ? p[j] * 0x1p24f : 0.f;
            }
          }
        }
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          typedef typename Tl::W W;
          const uint32_t h0 = W::down(y[2 * j]), h1 = W::down(y[2 * j + 1]);
          hi[j] = h0 | (h1 << 16);
          lo[j] = W::down(y[2 * j] - W::up(h0)) | (W::down(y[2 * j + 1] - W::up(h1)) << 16);
        }
        tile.template add_pair<0>(make_uint4(hi[0], hi[1], hi[2], hi[3]),
                                  make_uint4(lo[0], lo[1], lo[2], lo[3]), acc);
        if (!rest || lift == 0x1p48f) break;
        tile.transpose_again();
        lift *= 0x1p24f;
#pragma unroll
        for (int c = 0; c < Tl::kDims; ++c) acc[c] *= 0x1p24f;
      }
      if (lift != 1.f) {
        const float back = lift == 0x1p24f ? 0x1p-24f : 0x1p-48f;
#pragma unroll
        for (int c = 0; c < Tl::kDims; ++c) acc[c] *= back;
      }
      if (more) {
        load_v(off);
        now = next;
        if (tn + kWaves < t_end) next = octets_of(a, table, (tn + kWaves) * kTileKeys, n);
      }
      t = tn;
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // Join the wavefronts.
    __syncthreads();  // the last segment's readers are done
    if (g == 0) {
      ms[wave][l16] = m;
      ls[wave][l16] = l;
    }
    __syncthreads();
    float M = ms[0][l16];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) M = fmaxf(M, ms[i][l16]);
    const float mine = part_weight(m, M);
    if (l16 < heads) {
#pragma unroll
      for (int c = 0; c < Tl::kDims; c += 4)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4*>(&os[wave][l16][Tl::out_dim(4 * g + i, c)]) =
              make_float4(acc[c][i] * mine, acc[c + 1][i] * mine, acc[c + 2][i] * mine,
                          acc[c + 3][i] * mine);
    }
    __syncthreads();
    const bool full = s0 == 0 && s1 == row_slots;
    // Maximum and sum of query h over the wavefronts.
    auto join = [&](int h, float& M, float& L) {
      M = ms[0][h];
      for (int i = 1; i < kWaves; ++i) M = fmaxf(M, ms[i][h]);
      L = 0.f;
      for (int i = 0; i < kWaves; ++i)
        L += ls[i][h] * part_weight(ms[i][h], M);
    };
    float* part = a.parts + (int64_t)(2 * (w * Y + y) + (first_segment ? 0 : 1)) * a.part_floats;
    for (int x = tid; x < heads * (kDh / 4); x += kThreads) {
      const int h = x / (kDh / 4), d = 4 * (x % (kDh / 4));
      float4 o = *reinterpret_cast<const float4*>(&os[0][h][d]);
#pragma unroll
      for (int i = 1; i < kWaves; ++i) {
        const float4 e = *reinterpret_cast<const float4*>(&os[i][h][d]);
        o.x += e.x, o.y += e.y, o.z += e.z, o.w += e.w;
      }
      float M, L;
      if (full || d == 0) join(h, M, L);
      if (full) {
        store_out(grow, h, d, o, M, L);
      } else {
        uint64_t* p = reinterpret_cast<uint64_t*>(part + 32 + h * kDh + d);
        const uint64_t a0 = (uint64_t)__float_as_uint(o.x) | ((uint64_t)__float_as_uint(o.y) << 32);
        const uint64_t a1 = (uint64_t)__float_as_uint(o.z) | ((uint64_t)__float_as_uint(o.w) << 32);
        __hip_atomic_store(p, a0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(p + 1, a1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (d == 0) {
          st_u32<true>(part + h, __float_as_uint(M));
          st_u32<true>(part + 16 + h, __float_as_uint(L));
        }
      }
    }
    if (!full) {
      if (waiting == 0) shared0 = row;
      else shared1 = row;
      ++waiting;
    }
    u += s1 - s0;
    first_segment = false;
  }
  if (kWhole || waiting == 0) return;

  // The shared outputs, at most two: this worker's parts are in memory before
  // it takes their tickets, and whose ticket is the last joins the parts.
  wait_memory();
  __syncthreads();
  int base0, base1;
  const int end0 = slots_at(shared0, base0) + base0, end1 = slots_at(shared1, base1) + base1;
  if (tid < waiting) {
    const int base = tid ? base1 : base0, end = tid ? end1 : end0;
    const int wa = base / run, wb = (end - 1) / run;  // the first and the last worker
    last[tid] = __hip_atomic_fetch_add(&a.tickets[(wa * Y + y) * kTicketStride], 1u, __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(wb - wa);
    wait_memory();
  }
  __syncthreads();
  for (int turn = 0; turn < waiting; ++turn) {
    if (!last[turn]) continue;
    const int shared = turn ? shared1 : shared0, base = turn ? base1 : base0, end = turn ? end1 : end0;
    const int wa = base / run, parts = (end - 1) / run - wa + 1;
    const int lead = base % run ? 1 : 0;  // the first one's last segment, or its first
    auto part_at = [&](int i) {
      return a.parts + (int64_t)(2 * ((wa + i) * Y + y) + (i == 0 ? lead : 0)) * a.part_floats;
    };
    const int64_t grow = a.row0 + shared;
    // Eight parts at a time, everything of theirs in flight at once; the parts
    // are dealt over the threads that one part's outputs leave idle.
    const int items = heads * (kDh / 4);
    const int stripes = items < kThreads ? kThreads / items : 1;
    for (int x = tid; x < items * stripes; x += kThreads) {
      const int item = x % items, h = item / (kDh / 4), d = 4 * (item % (kDh / 4));
      float M = -INFINITY, L = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      constexpr int kAhead = 8;
      for (int i0 = x / items; i0 < parts; i0 += kAhead * stripes) {
        float m_of[kAhead], l_of[kAhead];
        uint64_t lo[kAhead], hi[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const float* p = part_at(min(i0 + k * stripes, parts - 1));
          const uint64_t* v = reinterpret_cast<const uint64_t*>(p + 32 + h * kDh + d);
          m_of[k] = __uint_as_float(ld_u32<true>(p + h));
          l_of[k] = __uint_as_float(ld_u32<true>(p + 16 + h));
          lo[k] = __hip_atomic_load(v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          hi[k] = __hip_atomic_load(v + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        float top = M;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          if (i0 + k * stripes >= parts) {  // past the end: nothing (an infinity times 0 is not)
            m_of[k] = -INFINITY;
            l_of[k] = 0.f;
            lo[k] = hi[k] = 0;
          }
          top = fmaxf(top, m_of[k]);
        }
        const float shrink = part_weight(M, top);
        M = top;
        L *= shrink;
        o.x *= shrink, o.y *= shrink, o.z *= shrink, o.w *= shrink;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const float f = part_weight(m_of[k], M);
          L = fmaf(f, l_of[k], L);
          o.x = fmaf(f, __uint_as_float((uint32_t)lo[k]), o.x);
          o.y = fmaf(f, __uint_as_float((uint32_t)(lo[k] >> 32)), o.y);
          o.z = fmaf(f, __uint_as_float((uint32_t)hi[k]), o.z);
          o.w = fmaf(f, __uint_as_float((uint32_t)(hi[k] >> 32)), o.w);
        }
      }
      if (stripes == 1) {
        store_out(grow, h, d, o, M, L);
      } else {
        striped[x] = o;
        striped_m[x] = M;
        striped_l[x] = L;
      }
    }
    if (stripes > 1) {
      __syncthreads();
      if (tid < items) {
        float M = striped_m[tid], L = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i = 1; i < stripes; ++i) M = fmaxf(M, striped_m[tid + i * items]);
        for (int x = tid; x < items * stripes; x += items) {
          const float f = part_weight(striped_m[x], M);
          const float4 e = striped[x];
          L = fmaf(f, striped_l[x], L);
          o.x = fmaf(f, e.x, o.x), o.y = fmaf(f, e.y, o.y);
          o.z = fmaf(f, e.z, o.z), o.w = fmaf(f, e.w, o.w);
        }
        store_out(grow, tid / (kDh / 4), 4 * (tid % (kDh / 4)), o, M, L);
      }
      __syncthreads();  // the next output's
    }
    if (tid == 0) st_u32<true>(&a.tickets[(wa * Y + y) * kTicketStride], 0);
  }
}

// ---------------------------------------------------------------- checks
int32_t check_kv(const emoe_paged_kv* kv) {
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

KvView view_of(const emoe_paged_kv& kv) {
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
int32_t check_io(const emoe_paged_kv& kv, int32_t dtype, const int32_t* table, int32_t n_seqs,
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

int32_t check_rows(const char* what, const void* p, int64_t stride, int64_t rows, int64_t width) {
  if (!p) return report_error(EMOE_EINVAL, "%s is NULL", what);
  if (!aligned16(p) || (rows > 1 && stride % 8))
    return report_error(EMOE_EINVAL, "%s: need 16-byte aligned rows", what);
  if (rows > 1 && stride < width)
    return report_error(EMOE_EINVAL, "%s: row stride %lld below the row's %lld elements", what,
                        (long long)stride, (long long)width);
  return EMOE_OK;
}

int32_t launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return report_error(EMOE_EHIP, "%s launch: %s", what, hipGetErrorString(e));
  return EMOE_OK;
}

template <class T, bool kE4M3>
void launch_append(const AppendArg& a, int head_dim, bool inter, dim3 grid, hipStream_t stream) {
#define APPEND_CASE(D)                                                                             \
  if (inter)                                                                                       \
    hipLaunchKernelGGL((paged_append_kernel<T, kE4M3, true, D>), grid, dim3(kThreads), 0, stream, a); \
  else                                                                                             \
    hipLaunchKernelGGL((paged_append_kernel<T, kE4M3, false, D>), grid, dim3(kThreads), 0, stream, a)
  if (head_dim == 64) {
    APPEND_CASE(64);
  } else if (head_dim == 128) {
    APPEND_CASE(128);
  } else {
    APPEND_CASE(256);
  }
#undef APPEND_CASE
}

template <class T, bool kE4M3>
void launch_attend(const AttendArg& a, int head_dim, int waves, hipStream_t stream) {
  const dim3 grid((unsigned)(a.workers * a.kv.n_kv_heads * a.q_tiles)), block(64 * waves);
#define ATTEND_CASE(D, W) \
  hipLaunchKernelGGL((paged_attention_kernel<T, kE4M3, D, W>), grid, block, 0, stream, a)
#define ATTEND_WAVES(D)                  \
  if (waves == 1) ATTEND_CASE(D, 1);     \
  else if (waves == 8) ATTEND_CASE(D, 8); \
  else ATTEND_CASE(D, 4)
  if (head_dim == 256) {
    if (waves == 1) ATTEND_CASE(256, 1);
    else ATTEND_CASE(256, 4);
  } else if (head_dim == 128) {
    ATTEND_WAVES(128);
  } else {
    ATTEND_WAVES(64);
  }
#undef ATTEND_WAVES
#undef ATTEND_CASE
}

// How a call is launched: rows per launch (their units stay below 2^31), the
// workers of each line (with one wavefront: its rows) and the lines (key heads
// times tiles of 16 queries), and the floats of one workgroup's record for a split output.
// The device holds 512 workgroups of four wavefronts, two to a CU, or 256 of eight
// (or of four at 256 dimensions: 65,536 keys of 4 heads 55 us, with 512 workers
// 67).  Eight join twice the keys in LDS that four do, which pays in two cases:
//  - with four, an output's parts would come to more than kWideJoin bytes, which
//    one workgroup reads: 131,072 keys of 8 heads 94 against 91 us, 8,192 keys
//    16.3 and 14.2, 4 rows of 4,000 keys of 4 heads with 8 queries each 17.4 and
//    13.9; below it 4 rows of 3,000 keys 17.1 and 17.6;
//  - there is a workgroup for every output, and what the idle ones could take
//    off the longest row comes to less than two units: 47 windows of 1,024 keys
//    14.5 and 12.7 us, 302 keys 9.6 and 9.0, 32 rows of 2,000 keys 50 and 45.7 (of
//    up to 2,000 25.4 and 27.0); above it 16 rows of up to 1,024 keys 12.9 and 17.
struct AttendPlan {
  int64_t rows_per_launch;
  int waves, workers, lines, part_floats;
  int64_t most_parts;  // workgroups of any plan with these rows, heads and max_keys
};
// One wavefront, a workgroup to every output, where a row has a tile or two (no
// more than kShortKeys keys: one row of 10 6.3 -> 4.4 us, 282 of up to 30 21 ->
// 7.9; above, 4 rows of 128 7.3 and 8.2), or up to kManyKeys with more outputs
// than the device holds workgroups twice over (1,600 outputs of up to 250 keys
// 29 -> 19.8 us, of up to 500 37.6 -> 34.7; of up to 1,000 62 and 65.5, 512
// outputs of up to 250 11 and 13.6): the wavefronts that a short row leaves idle
// take other rows, and nothing is planned.
constexpr int kPlaces = 512, kWideJoin = 96 << 10, kShortKeys = 64, kManyKeys = 512;
constexpr int kMostWhole = 1 << 20;  // outputs: a grid below 2^32 threads
AttendPlan attend_plan(const emoe_paged_kv& kv, int32_t rows, int32_t n_heads, int32_t max_keys,
                       int32_t window) {
  const int group = n_heads / kv.n_kv_heads;
  const int64_t keys = window > 0 && window < max_keys ? window : max_keys;
  AttendPlan p;
  p.lines = kv.n_kv_heads * ((group + 15) / 16);
  const int record = 4 * (group < 16 ? group : 16) * kv.head_dim;
  const int64_t outputs = (int64_t)rows * p.lines, four = 4 * kTileKeys, eight = 8 * kTileKeys;
  int64_t parts = outputs > 0 ? kPlaces / outputs : 0;
  if (parts > (keys + four - 1) / four) parts = (keys + four - 1) / four;
  const int64_t idle = kPlaces / 2 - outputs;
  const bool whole = idle >= 0 && (keys + eight - 1) / eight * idle < kPlaces;
  if (outputs <= kMostWhole && (keys <= kShortKeys || (keys <= kManyKeys && outputs > 2 * kPlaces)))
    p.waves = 1;
  else
    p.waves = kv.head_dim < 256 && (whole || parts * record > kWideJoin) ? 8 : 4;
  const int64_t most = keys / (kTileKeys * p.waves) + 2;  // units of one row
  p.rows_per_launch = (((int64_t)1 << 31) - 1 - kTickets) / most;
  if (p.rows_per_launch > kMaxRows) p.rows_per_launch = kMaxRows;
  const int64_t held = rows < p.rows_per_launch ? rows : p.rows_per_launch;
  int64_t workers = (kv.head_dim == 256 || p.waves == 8 ? kPlaces / 2 : kPlaces) / p.lines;
  if (workers < 1) workers = 1;
  p.workers = (int)(held * most < workers ? held * most : workers);
  p.part_floats = 32 + (group < 16 ? group : 16) * kv.head_dim;
  p.most_parts = p.lines > kPlaces ? p.lines : kPlaces;
  return p;
}

// Bounds of the calls' integers: keys of a row and what a tile adds to them stay
// within 32 bits, and lines times threads within a grid; an appended token's
// items (at most 2^24 of q and, as a page's slots are below 2^30 elements, 2^27 of
// k and v) and what a step of its workgroups adds to them stay within 32 bits.
constexpr int32_t kMostKeys = 1 << 30, kMostHeads = 1 << 20;

}  // namespace

extern "C" {

int32_t emoe_check_paged_kv(const emoe_paged_kv* kv) { return check_kv(kv); }

int32_t emoe_paged_append(const emoe_paged_kv* kv, const emoe_paged_append_args* args,
                          hipStream_t stream) {
  int32_t st = check_kv(kv);
  if (st) return st;
  if (!args) return report_error(EMOE_EINVAL, "args is NULL");
  const emoe_paged_append_args& A = *args;
  if ((st = check_io(*kv, A.dtype, A.page_table, A.n_seqs, A.table_width, A.table_stride))) return st;
  if (A.tokens < 0) return report_error(EMOE_EINVAL, "tokens %d", A.tokens);
  if (A.rotary_dim < 0 || A.rotary_dim > kv->head_dim || A.rotary_dim % 16)
    return report_error(EMOE_ESHAPE, "rotary_dim %d: need a multiple of 16 up to head_dim %d",
                        A.rotary_dim, kv->head_dim);
  if (A.interleaved != 0 && A.interleaved != 1)
    return report_error(EMOE_EINVAL, "interleaved %d: need 0 or 1", A.interleaved);
  if (A.q && (A.n_heads < 1 || A.n_heads > kMostHeads))
    return report_error(EMOE_ESHAPE, "n_heads %d: need 1 to 2^20", A.n_heads);
  if (A.tokens == 0) return EMOE_OK;
  const int64_t dh = kv->head_dim, kw = kv->n_kv_heads * dh, qw = (int64_t)A.n_heads * dh;
  if (A.rotary_dim > 0 && !A.inv_freq) return report_error(EMOE_EINVAL, "inv_freq is NULL");
  if (!A.positions) return report_error(EMOE_EINVAL, "positions is NULL");
  if ((st = check_rows("k", A.k, A.k_stride, A.tokens, kw))) return st;
  if ((st = check_rows("v", A.v, A.v_stride, A.tokens, kw))) return st;
  if (A.q) {
    if ((st = check_rows("q", A.q, A.q_stride, A.tokens, qw))) return st;
    if ((st = check_rows("q_out", A.q_out, A.q_out_stride, A.tokens, qw))) return st;
  }
  AppendArg a;
  a.kv = view_of(*kv);
  a.q = static_cast<const uint16_t*>(A.q);
  a.k = static_cast<const uint16_t*>(A.k);
  a.v = static_cast<const uint16_t*>(A.v);
  a.q_out = static_cast<uint16_t*>(A.q_out);
  a.positions = A.positions;
  a.seqs = A.seqs;
  a.table = A.page_table;
  a.inv_freq = A.inv_freq;
  a.q_stride = A.q_stride;
  a.k_stride = A.k_stride;
  a.v_stride = A.v_stride;
  a.qo_stride = A.q_out_stride;
  a.table_stride = A.table_stride;
  a.n_heads = A.n_heads;
  a.n_seqs = A.n_seqs;
  a.table_width = A.table_width;
  a.rotary_dim = A.rotary_dim;
  const int64_t heads = (A.q ? A.n_heads : 0) + 2 * (int64_t)kv->n_kv_heads;
  const int64_t items = heads * (dh / 16);
  int64_t gy = 1;  // small calls: up to an item per thread
  while (A.tokens * gy < 512 && gy * kThreads < items) ++gy;
  const bool e4m3 = kv->dtype == EMOE_E4M3, inter = A.interleaved != 0;
  constexpr int64_t kTokens = 1 << 22;  // of one launch: a grid has fewer than 2^32 threads
  for (a.token0 = 0; a.token0 < A.tokens; a.token0 += kTokens) {
    const int64_t gx = A.tokens - a.token0 < kTokens ? A.tokens - a.token0 : kTokens;
    const dim3 grid((unsigned)gx, (unsigned)gy);
    if (A.dtype == EMOE_BF16) {
      if (e4m3) launch_append<Bf16, true>(a, kv->head_dim, inter, grid, stream);
      else launch_append<Bf16, false>(a, kv->head_dim, inter, grid, stream);
    } else {
      if (e4m3) launch_append<Fp16, true>(a, kv->head_dim, inter, grid, stream);
      else launch_append<Fp16, false>(a, kv->head_dim, inter, grid, stream);
    }
    if ((st = launched("paged_append_kernel"))) return st;
  }
  return EMOE_OK;
}

size_t emoe_paged_attention_workspace_bytes(const emoe_paged_kv* kv, int32_t rows, int32_t n_heads,
                                            int32_t max_keys) {
  if (check_kv(kv) || rows < 0 || n_heads < 1 || n_heads % kv->n_kv_heads || max_keys < 0 ||
      max_keys > kMostKeys || n_heads > kMostHeads)
    return 0;
  const AttendPlan p = attend_plan(*kv, rows, n_heads, max_keys, 0);
  return EMOE_SERVING_TICKET_BYTES + (size_t)2 * p.most_parts * p.part_floats * 4;
}

int32_t emoe_paged_attention(const emoe_paged_kv* kv, const emoe_paged_attention_args* args,
                             void* workspace, size_t workspace_bytes, hipStream_t stream) {
  int32_t st = check_kv(kv);
  if (st) return st;
  if (!args) return report_error(EMOE_EINVAL, "args is NULL");
  const emoe_paged_attention_args& A = *args;
  if ((st = check_io(*kv, A.dtype, A.page_table, A.n_seqs, A.table_width, A.table_stride))) return st;
  if (A.rows < 0 || A.max_keys < 0 || A.window < 0)
    return report_error(EMOE_EINVAL, "negative rows, max_keys or window (%d, %d, %d)", A.rows,
                        A.max_keys, A.window);
  if (A.n_heads < 1 || A.n_heads % kv->n_kv_heads)
    return report_error(EMOE_ESHAPE, "n_heads %d is no multiple of n_kv_heads %d", A.n_heads,
                        kv->n_kv_heads);
  if (A.max_keys > kMostKeys || A.n_heads > kMostHeads)
    return report_error(EMOE_ESHAPE, "max_keys %d or n_heads %d: need at most 2^30 and 2^20", A.max_keys,
                        A.n_heads);
  if (!std::isfinite(A.scale * 1.4426950408889634f))  // as the kernel takes it
    return report_error(EMOE_EINVAL, "scale %g is not finite, or near the largest number", A.scale);
  if (A.rows == 0) return EMOE_OK;
  const int64_t qw = (int64_t)A.n_heads * kv->head_dim;
  if ((st = check_rows("q", A.q, A.q_stride, A.rows, qw))) return st;
  if ((st = check_rows("out", A.out, A.out_stride, A.rows, qw))) return st;
  if (!A.lengths) return report_error(EMOE_EINVAL, "lengths is NULL");
  const size_t need = emoe_paged_attention_workspace_bytes(kv, A.rows, A.n_heads, A.max_keys);
  if (!workspace || workspace_bytes < need)
    return report_error(EMOE_EINVAL, "workspace of %zu bytes < %zu needed", workspace ? workspace_bytes : 0,
                        need);
  if (!aligned16(workspace)) return report_error(EMOE_EINVAL, "workspace: need 16-byte alignment");
  const AttendPlan plan = attend_plan(*kv, A.rows, A.n_heads, A.max_keys, A.window);
  AttendArg a;
  a.kv = view_of(*kv);
  a.q = static_cast<const uint16_t*>(A.q);
  a.out = static_cast<uint16_t*>(A.out);
  a.lse = A.lse;
  a.lengths = A.lengths;
  a.seqs = A.seqs;
  a.table = A.page_table;
  a.tickets = static_cast<uint32_t*>(workspace);
  a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + EMOE_SERVING_TICKET_BYTES);
  a.q_stride = A.q_stride;
  a.out_stride = A.out_stride;
  a.table_stride = A.table_stride;
  a.scale = A.scale;
  a.n_heads = A.n_heads;
  a.group = A.n_heads / kv->n_kv_heads;
  a.q_tiles = (a.group + 15) / 16;
  a.n_seqs = A.n_seqs;
  a.table_width = A.table_width;
  a.max_keys = A.max_keys;
  a.window = A.window;
  a.part_floats = plan.part_floats;
  const bool e4m3 = kv->dtype == EMOE_E4M3;
  for (int64_t r0 = 0; r0 < A.rows; r0 += plan.rows_per_launch) {
    a.row0 = (int32_t)r0;
    a.rows = (int32_t)(A.rows - r0 < plan.rows_per_launch ? A.rows - r0 : plan.rows_per_launch);
    a.workers = plan.waves == 1 ? a.rows : plan.workers;
    if (A.dtype == EMOE_BF16) {
      if (e4m3) launch_attend<Bf16, true>(a, kv->head_dim, plan.waves, stream);
      else launch_attend<Bf16, false>(a, kv->head_dim, plan.waves, stream);
    } else {
      if (e4m3) launch_attend<Fp16, true>(a, kv->head_dim, plan.waves, stream);
      else launch_attend<Fp16, false>(a, kv->head_dim, plan.waves, stream);
    }
    if ((st = launched("paged_attention_kernel"))) return st;
  }
  return EMOE_OK;
}

}  // extern "C"
