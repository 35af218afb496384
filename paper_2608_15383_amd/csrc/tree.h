// The attention of trees of drafted tokens over a paged cache
// (exactmoe_drafts.h): its kernels, which tree_bf16.hip and tree_fp16.hip build for
// their types.
#pragma once

#include "exactmoe_drafts.h"
#include "paged.h"

namespace emoe {

struct TreeArg {
  KvView kv;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  const int32_t *lengths, *starts, *seqs, *table;
  const uint64_t* tree;
  const float* slopes;
  int32_t* heads_of;  // of each output that workgroups share: first worker, parts, place in its first
  float* parts;
  int64_t q_stride, out_stride, table_stride;
  float scale, cap;
  int32_t tree0, trees, rows, n_heads, group, blocks, n_seqs, table_width, max_keys, max_nodes, window;
  int32_t workers, slack;  // workers 0: a workgroup to every output
  int32_t unit_keys, unit_log2;
  int32_t part_floats;
};

// How a call is launched (tree.hip chooses): the tiles of 16 columns of a block, and the
// rest as in TreeArg.
struct TreePlan {
  int64_t trees_per_launch;
  bool wide;  // paged_tree_wide_kernel
  int tiles, blocks, lines, workers, slack, part_floats, stripes, unit_keys;
  int64_t most_parts, most_shared;
};

void launch_tree_bf16(const TreeArg& a, const TreePlan& p, int head_dim, bool e4m3, hipStream_t stream);
void launch_tree_fp16(const TreeArg& a, const TreePlan& p, int head_dim, bool e4m3, hipStream_t stream);

constexpr int kTreeWaves = 4;

// Workgroups of paged_tree_wide_kernel on a CU.  128 dimensions over 8 bits: 40 trees 173 us with
// two and 163 with three, which leave 168 registers and so 1 value in scratch memory, 14 with shaped
// scores.  64 dimensions over 16 bits 34.5 with three and 40.9 with four (16 trees of up to 8,192
// keys).  Of 256 dimensions two share the 512 registers, with 12 values in scratch memory under
// shaped scores (fp16 over 16 bits 27, and 7 without); one alone has not been measured.
constexpr int wide_workgroups(int head_dim, bool e4m3) {
  return head_dim == 64 || (head_dim == 128 && e4m3) ? 3 : 2;
}

// Its steps' tiles of 32 keys: 33 trees with scores by distance, 64 dimensions over 16 bits,
// 34 us with one and 40 with two.
constexpr int wide_step_tiles(int head_dim, bool e4m3) { return !e4m3 && head_dim != 128 ? 1 : 2; }

// A tree: its rows, and the keys [first, end) that some node of it may see, of
// which those from n on are its nodes.
struct TreeSpan {
  int start, count, seq, n, first, end;
};
__device__ __forceinline__ TreeSpan tree_span(const TreeArg& a, int g) {
  TreeSpan s;
  const int length = a.lengths[g];
  int next = 0;
  s.start = g * a.max_nodes;
  s.seq = g;
  if (a.starts) {
    s.start = a.starts[g];
    next = a.starts[g + 1];
  }
  if (a.seqs) s.seq = a.seqs[g];
  const int64_t count = a.starts ? (int64_t)next - s.start : a.max_nodes;
  if (s.start < 0 || s.start > a.rows) s.start = a.rows;
  s.count = (int)max((int64_t)0, min(count, (int64_t)min(a.max_nodes, a.rows - s.start)));
  s.n = min(length, 1 << 30);
  s.first = s.end = 0;
  if ((uint32_t)s.seq < (uint32_t)a.n_seqs && s.n >= 0) {
    const int64_t most = min((int64_t)a.max_keys, (int64_t)a.table_width << a.kv.page_log2);
    s.end = (int)min((int64_t)s.n + s.count, most);
    s.first = a.window > 0 ? min(s.end, max(0, s.n + 1 - a.window)) : 0;
  }
  return s;
}
// Units (of unit_keys keys) of each of its column blocks; a tree that sees no key has
// one, which writes its zeros.
__device__ __forceinline__ int tree_units(const TreeArg& a, const TreeSpan& s) {
  return max(1, ((s.end + a.unit_keys - 1) >> a.unit_log2) - (s.first >> a.unit_log2));
}

// x = cap * tanh(x / cap), to a few units of fp32's rounding: below 0.3 by tanh's
// series (1 - 2 / (1 + e^2y) would cancel), which alone serves a wavefront whose
// scores are all that small beside the cap.
template <int kKeys>
__device__ __forceinline__ void cap_scores(float (&x)[kKeys], float cap, float inv_cap) {
  float most = 0.f;
#pragma unroll
  for (int j = 0; j < kKeys; ++j) {
    x[j] *= inv_cap;
    most = fmaxf(most, fabsf(x[j]));
  }
  float far[kKeys];
  const bool any_far = __any(!(most < 0.3f));
  if (any_far) {
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
      const float t = exp2_hw(fabsf(x[j]) * -2.8853900817779268f);
      far[j] = copysignf((1.f - t) * __builtin_amdgcn_rcpf(1.f + t), x[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < kKeys; ++j) {
    const float y = x[j], z = y * y;
    float s = fmaf(z, 21844.f / 6081075.f, -1382.f / 155925.f);
    s = fmaf(z, s, 62.f / 2835.f);
    s = fmaf(z, s, -17.f / 315.f);
    s = fmaf(z, s, 2.f / 15.f);
    s = fmaf(z, s, -1.f / 3.f);
    const float near = fmaf(y * z, s, y);
    x[j] = cap * (any_far && !(fabsf(y) < 0.3f) ? far[j] : near);
  }
}

// Lane group kg's weight j of each column.
template <int kKeys>
__device__ __forceinline__ float weight_of(const float (&p)[kKeys], int j, int kg) {
  float own = p[0];
#pragma unroll
  for (int k = 1; k < kKeys; ++k) own = j == k ? p[k] : own;
  return __shfl(own, 16 * kg + (lane_id() & 15));
}
// sum + weight * v where the column sees it.
__device__ __forceinline__ f32x4 add_where(bool sees, float weight, const f32x4& v, const f32x4& sum) {
  f32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = sees ? fmaf(weight, v[i], sum[i]) : sum[i];
  return r;
}

// Tile (paged.h) for kTiles tiles of 16 columns, so that what is made of keys and
// values (trades between lanes, conversions, transposes) is made once for all.
template <class T, bool kE4M3, int kDh, int kTiles>
struct WideTile : Tile<T, kE4M3, kDh> {
  typedef Tile<T, kE4M3, kDh> B;
  typedef typename B::H16 H16;
  typedef typename B::HW HW;

  __device__ __forceinline__ void wide_scores(const uint4 (&q)[kTiles][B::kSteps], bool second,
                                              f32x4 (&s)[kTiles][2]) const {
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) s[n][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < B::kPairs; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t c0[B::kChunkWords], c1[B::kChunkWords];
#pragma unroll
        for (int w = 0; w < B::kChunkWords; ++w) {
          const uint32_t a = this->k[2 * h][p][w], b = this->k[2 * h + 1][p][w];
          const uint32_t a2 = __builtin_amdgcn_update_dpp(0, (int)a, 0x4E, 0xF, 0xF, true);
          const uint32_t b2 = __builtin_amdgcn_update_dpp(0, (int)b, 0x4E, 0xF, 0xF, true);
          c0[w] = second ? b2 : a;
          c1[w] = second ? b : a2;
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int sub = 0; sub < B::kSub; ++sub) {
            const uint32_t(&c)[B::kChunkWords] = half ? c1 : c0;
            uint4 x;
            if constexpr (kE4M3) {
              const uint32_t lo = c[2 * sub], hi = c[2 * sub + 1];
              x = make_uint4(H16::template from_e4m3<false>(lo), H16::template from_e4m3<true>(lo),
                             H16::template from_e4m3<false>(hi), H16::template from_e4m3<true>(hi));
            } else {
              x = make_uint4(c[0], c[1], c[2], c[3]);
            }
#pragma unroll
            for (int n = 0; n < kTiles; ++n)
              s[n][h] = H16::mfma(x, q[n][(2 * p + half) * B::kSub + sub], s[n][h]);
          }
      }
  }

  template <int kW>
  __device__ __forceinline__ void wide_add(const uint4 (&hi)[kTiles][1], const uint4 (&lo)[kTiles][1],
                                           f32x4 (&acc)[kTiles][B::kDims]) const {
    uint32_t e[4], o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = this->template pair<kW>(2 * i), b = this->template pair<kW>(2 * i + 1);
      e[i] = __builtin_amdgcn_perm(b, a, 0x05040100u);
      o[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    }
    const uint4 ve = make_uint4(e[0], e[1], e[2], e[3]), vo = make_uint4(o[0], o[1], o[2], o[3]);
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      acc[n][2 * kW] = HW::mfma(ve, hi[n][0], acc[n][2 * kW]);
      acc[n][2 * kW + 1] = HW::mfma(vo, hi[n][0], acc[n][2 * kW + 1]);
    }
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      acc[n][2 * kW] = HW::mfma(ve, lo[n][0], acc[n][2 * kW]);
      acc[n][2 * kW + 1] = HW::mfma(vo, lo[n][0], acc[n][2 * kW + 1]);
    }
    if constexpr (kW + 1 < B::kDims / 2) wide_add<kW + 1>(hi, lo, acc);
  }

  // Adds the values of the lanes' key j, of one lane group alone (`here`), times the
  // columns' weights to those that see it: a weight of 1 brings them to the output's lanes.
  template <int kW>
  __device__ __forceinline__ void add_key(int j, bool here, const float (&weight)[kTiles],
                                          const bool (&sees_it)[kTiles], f32x4 (&acc)[kTiles][B::kDims]) const {
    constexpr uint32_t kOne = B::kF16Weights ? 0x3c00u : 0x3f80u;
    uint32_t e[4], o[4], ones[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = this->template pair<kW>(2 * i), b = this->template pair<kW>(2 * i + 1);
      const uint32_t mask = here && (j >> 1) == i ? (j & 1 ? 0xffff0000u : 0xffffu) : 0u;
      e[i] = __builtin_amdgcn_perm(b, a, 0x05040100u) & mask;
      o[i] = __builtin_amdgcn_perm(b, a, 0x07060302u) & mask;
      ones[i] = (kOne | kOne << 16) & mask;
    }
    const uint4 one = make_uint4(ones[0], ones[1], ones[2], ones[3]);
    const f32x4 ve = HW::mfma(make_uint4(e[0], e[1], e[2], e[3]), one, f32x4{0.f, 0.f, 0.f, 0.f});
    const f32x4 vo = HW::mfma(make_uint4(o[0], o[1], o[2], o[3]), one, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
      acc[n][2 * kW] = add_where(sees_it[n], weight[n], ve, acc[n][2 * kW]);
      acc[n][2 * kW + 1] = add_where(sees_it[n], weight[n], vo, acc[n][2 * kW + 1]);
    }
    if constexpr (kW + 1 < B::kDims / 2) add_key<kW + 1>(j, here, weight, sees_it, acc);
  }

  // Whether any of a lane's values is infinite or NaN: an exponent of all ones carries.
  __device__ __forceinline__ bool any_not_finite() const {
    constexpr uint32_t kAbs = kE4M3 ? 0x7f7f7f7fu : 0x7fff7fffu;
    constexpr uint32_t kOne = kE4M3 ? 0x01010101u : T::kType == EMOE_F16 ? 0x04000400u : 0x00800080u;
    uint32_t any = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int w = 0; w < B::kVWords; ++w) any |= (this->v[j][w] & kAbs) + kOne;
    return (any & ~kAbs) != 0;
  }
  // Which of its 8 keys have such a value.
  __device__ __forceinline__ uint32_t not_finite() const {
    constexpr uint32_t kAbs = kE4M3 ? 0x7f7f7f7fu : 0x7fff7fffu;
    constexpr uint32_t kOne = kE4M3 ? 0x01010101u : T::kType == EMOE_F16 ? 0x04000400u : 0x00800080u;
    uint32_t bad = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t any = 0;
#pragma unroll
      for (int w = 0; w < B::kVWords; ++w) any |= (this->v[j][w] & kAbs) + kOne;
      bad |= (any & ~kAbs) != 0 ? 1u << j : 0u;
    }
    return bad;
  }
};

// The scores of a tile in powers of two: capped, and less the bias by distance.
// key_at[j] is the key's place from the tree's first node on: below 0 its position,
// else (only if `nodes`) the node, whose depth is in that lane.
template <int kTiles, int kKeys>
__device__ __forceinline__ void shape_scores(float (&z)[kTiles][kKeys], float cap, float inv_cap, bool biased,
                                             const float (&slope)[kTiles], const int (&deep_at)[kTiles],
                                             int (&key_at)[kKeys], bool nodes, int depth) {
  if (cap > 0.f) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) cap_scores(z[i], cap, inv_cap);
  }
  if (biased && nodes) {
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
      const int deep = __shfl(depth, key_at[j] & 63);
      key_at[j] = key_at[j] < 0 ? key_at[j] : deep;
    }
  }
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
      z[i][j] *= 1.4426950408889634f;
      if (biased) z[i][j] = fmaf(-slope[i], (float)abs(deep_at[i] - key_at[j]), z[i][j]);
    }
}

// Which of the keys key0 .. key0 + 31 there are: within [first, end), in an octet that
// has a page (4 bits).
__device__ __forceinline__ uint32_t keys_there(int key0, int first, int end, uint32_t octets) {
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) bits |= octets >> i & 1 ? 0xffu << (8 * i) : 0u;
  if (first > key0) bits &= first - key0 > 31 ? 0u : ~0u << (first - key0);
  if (end - key0 < 32) bits &= end <= key0 ? 0u : (1u << (end - key0)) - 1;
  return bits;
}
// Which of them a node of this mask and depth sees, the tree's nodes being the keys from
// n on; depth: that of node i in lane i.
__device__ __forceinline__ uint32_t keys_seen(int key0, int n, uint64_t mask, int deep, int window, int depth) {
  const int old = n - key0;  // keys before the tree
  uint32_t bits = old >= 32 ? ~0u : old > 0 ? (uint32_t)(mask << old) | ((1u << old) - 1)
                                  : -old < 64 ? (uint32_t)(mask >> -old) : 0u;
  if (window > 0) {
    const int low = old + deep - window + 1;  // the first old key within the window
    const uint32_t nodes = old >= 32 ? 0u : old > 0 ? ~0u << old : ~0u;
    bits &= nodes | (low > 31 ? 0u : low > 0 ? ~0u << low : ~0u);
    if (window < 64) {
#pragma unroll 1
      for (int b = max(0, old); b < 32 && b - old < 64; ++b)
        if (__builtin_amdgcn_readlane(depth, b - old) <= deep - window) bits &= ~(1u << b);
    }
  }
  return bits;
}

// One tile's step of the softmax: weights p of the scores z, which a factor >= 0 makes
// powers of two.  The exponent m that a column's weights refer to is that of the
// maximum of its first tile (plus 2^lead), and follows the maximum again only when the
// weights of a lane come to more than 2^(8 + lead): until then nothing is rescaled, and
// no maximum sought.  fp16 weights begin at 2^7: there is room above, but little below.
// In a tile with masked keys, of score -inf, those weigh 0 even if the factor is 0.
template <class Tl, int kTiles, int kAcc, int kKeys>
__device__ __forceinline__ void soft_step(const float (&z)[kTiles][kKeys], float factor, bool masked,
                                          float (&m)[kTiles], float (&l)[kTiles],
                                          f32x4 (&acc)[kTiles][kAcc], float (&p)[kTiles][kKeys]) {
  constexpr float kLead = Tl::kF16Weights ? 7.f : 0.f;
  float sum[kTiles];
  auto weights = [&](int i) __attribute__((always_inline)) {
    const float ref = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
    for (int j = 0; j < kKeys; ++j) p[i][j] = exp2_hw(fmaf(z[i][j], factor, -ref));
    if (masked) {
#pragma unroll
      for (int j = 0; j < kKeys; ++j) p[i][j] = z[i][j] == -INFINITY ? 0.f : p[i][j];
    }
    float s[4] = {p[i][0], p[i][1], p[i][2], p[i][3]};
#pragma unroll
    for (int j = 4; j < kKeys; ++j) s[j & 3] += p[i][j];
    sum[i] = (s[0] + s[1]) + (s[2] + s[3]);
  };
  bool follow = false;
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    weights(i);
    follow = follow || m[i] == -INFINITY || sum[i] > (Tl::kF16Weights ? 0x1p15f : 0x1p8f);
  }
  if (__any(follow)) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      float top = z[i][0];
#pragma unroll
      for (int j = 1; j < kKeys; ++j) top = fmaxf(top, z[i][j]);
      top *= factor;
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m2 = fmaxf(m[i], top - kLead);
      const float shrink = m2 == -INFINITY ? 0.f : exp2_hw(m[i] - m2);
      m[i] = m2;
      l[i] *= shrink;
#pragma unroll
      for (int c = 0; c < kAcc; ++c) acc[i][c] *= shrink;
      weights(i);
    }
  }
#pragma unroll
  for (int i = 0; i < kTiles; ++i) l[i] += sum[i];
}

// Two values rounded to a pair of the type, and up again.
__device__ __forceinline__ uint32_t pair_down(Bf16, float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint32_t pair_down(Fp16, float a, float b) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  const f16x2 v = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float pair_up(Bf16, uint32_t w, bool high) {
  return __uint_as_float(high ? w & 0xffff0000u : w << 16);
}
__device__ __forceinline__ float pair_up(Fp16, uint32_t w, bool high) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  const f16x2 v = __builtin_bit_cast(f16x2, w);
  return (float)(high ? v.y : v.x);
}

// Adds the weighted values by add(high halves, low halves).  Weights as two 16-bit halves; small fp16 weights in turns
// of their own, 2^24 and 2^48 times as large, as in paged_attention_kernel.
template <class Tl, int kTiles, int kAcc, int kKeys, class Add>
__device__ __forceinline__ void add_in_halves(float (&p)[kTiles][kKeys], f32x4 (&acc)[kTiles][kAcc], Add add) {
  typedef typename Tl::W W;
  float lift = 1.f;
  while (true) {
    bool rest = false;
    float part[kTiles][kKeys];
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int j = 0; j < kKeys; ++j) part[i][j] = p[i][j];
    if constexpr (Tl::kF16Weights) {
      uint32_t least = ~0u;  // the bits, less 1, of the smallest weight above 0
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int j = 0; j < kKeys; ++j) least = min(least, __float_as_uint(p[i][j]) - 1u);
      rest = __any(least < __float_as_uint(0x1p-9f) - 1u);
      if (rest) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int j = 0; j < kKeys; ++j) {
            const bool small = p[i][j] < 0x1p-9f;
            part[i][j] = small ? 0.f : p[i][j];
            p[i][j] = small ? p[i][j] * 0x1p24f : 0.f;
          }
      }
    }
    uint4 hi[kTiles][kKeys / 8], lo[kTiles][kKeys / 8];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      uint32_t h[kKeys / 2], r[kKeys / 2];
#pragma unroll
      for (int j = 0; j < kKeys / 2; ++j) {
        h[j] = pair_down(W(), part[i][2 * j], part[i][2 * j + 1]);
        asm("" : "+v"(h[j]));  // one conversion of the pair, not a further one of each
        r[j] = pair_down(W(), part[i][2 * j] - pair_up(W(), h[j], false),
                         part[i][2 * j + 1] - pair_up(W(), h[j], true));
      }
#pragma unroll
      for (int k = 0; k < kKeys / 8; ++k) {
        hi[i][k] = make_uint4(h[4 * k], h[4 * k + 1], h[4 * k + 2], h[4 * k + 3]);
        lo[i][k] = make_uint4(r[4 * k], r[4 * k + 1], r[4 * k + 2], r[4 * k + 3]);
      }
    }
    add(hi, lo);
    if (!rest || lift == 0x1p48f) break;
    lift *= 0x1p24f;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int c = 0; c < kAcc; ++c) acc[i][c] *= 0x1p24f;
  }
  if (lift != 1.f) {
    const float back = lift == 0x1p24f ? 0x1p-24f : 0x1p-48f;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int c = 0; c < kAcc; ++c) acc[i][c] *= back;
  }
}

// A query's chunk, its sign turned where the scores' scale is negative (so that the
// scale may be taken as positive).
__device__ __forceinline__ uint4 signed_chunk(const uint16_t* at, uint32_t flip) {
  const uint4 x = *reinterpret_cast<const uint4*>(at);
  return make_uint4(x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip);
}

// The trees of a chunk of 64, one per lane.
struct TreeChunk {
  TreeSpan span;
  int first, units, blocks;

  __device__ __forceinline__ void load(const TreeArg& a, int c0, int columns) {
    first = c0;
    units = blocks = 0;
    span = TreeSpan{0, 0, 0, 0, 0, 0};
    if (c0 + lane_id() < a.trees) {
      span = tree_span(a, a.tree0 + c0 + lane_id());
      units = tree_units(a, span);
      blocks = (span.count * a.group + columns - 1) / columns;
    }
  }
};

// How the blocks of a launch are cut for the workers of a key head.  Either a block has
// ceil(units / target) parts and every worker one, so that a worker never begins a
// second block, which costs it as much as several units; or, where there are too few
// workers for that, or more trees than the 64 that a wavefront holds a lane each, the units
// of all blocks stand behind each other and every worker takes the same number of them.
// Parts and equal runs: 64 trees of 2 key heads over up to 16,384 keys 71 and 89 us (8 nodes), 65
// and 70 (2), 4 trees of 64 nodes over 8,192 83 and 103; 100 trees of 8 nodes take 125, in runs.
struct TreeRun {
  int u, u_end, base;    // units: of the run, the first one of block cb of tree tr
  int tr, cb;
  int run, each;         // units of a run; of a part (0: equal runs)
};
__device__ __forceinline__ bool find_run(const TreeArg& a, int w, int columns, TreeChunk& ch, TreeRun& r) {
  int total = 0;
  for (int c0 = 0; c0 < a.trees; c0 += 64) {
    ch.load(a, c0, columns);
    total += __builtin_amdgcn_readlane(wave_scan(ch.units * ch.blocks), 63);
  }
  r.run = (total + a.workers - 1) / a.workers;
  r.each = 0;
  r.base = 0;
  if (a.trees <= 64) {
    for (int t = r.run; t <= r.run + a.slack; t += max(1, t / 8)) {
      const int parts = ch.blocks ? (int)((uint32_t)(ch.units + t - 1) / (uint32_t)t) : 0;
      const int own = parts * ch.blocks, incl = wave_scan(own);
      const int all = __builtin_amdgcn_readlane(incl, 63);
      if (all > a.workers) continue;
      if (w >= all) return false;
      const int i = (int)__builtin_ctzll(__ballot(w < incl));
      const int units = __builtin_amdgcn_readlane(ch.units, i), cuts = __builtin_amdgcn_readlane(parts, i);
      const int at = w - __builtin_amdgcn_readlane(incl - own, i);
      r.tr = i;
      r.cb = at / cuts;
      r.each = (int)((uint32_t)(units + cuts - 1) / (uint32_t)cuts);
      r.u = (at % cuts) * r.each;
      r.u_end = min(units, r.u + r.each);
      return r.u < r.u_end;
    }
  }
  if ((int64_t)w * r.run >= total) return false;
  r.u = w * r.run;
  r.u_end = min(r.u + r.run, total);
  for (int c0 = 0;; c0 += 64) {
    if (a.trees > 64) ch.load(a, c0, columns);
    const int own = ch.units * ch.blocks, incl = wave_scan(own);
    const int all = __builtin_amdgcn_readlane(incl, 63);
    if (r.u < r.base + all) {
      const int i = (int)__builtin_ctzll(__ballot(r.u < r.base + incl));
      r.base += __builtin_amdgcn_readlane(incl - own, i);
      const int units = __builtin_amdgcn_readlane(ch.units, i);
      r.cb = (r.u - r.base) / units;
      r.base += r.cb * units;
      r.tr = c0 + i;
      return true;
    }
    r.base += all;
  }
}
// All of it the same for the whole wavefront, which the compiler does not see of loops
// whose ends depend on other lanes' values.
__device__ __forceinline__ void make_uniform(TreeRun& r) {
  r.u = __builtin_amdgcn_readfirstlane(r.u);
  r.u_end = __builtin_amdgcn_readfirstlane(r.u_end);
  r.base = __builtin_amdgcn_readfirstlane(r.base);
  r.tr = __builtin_amdgcn_readfirstlane(r.tr);
  r.cb = __builtin_amdgcn_readfirstlane(r.cb);
  r.run = __builtin_amdgcn_readfirstlane(r.run);
  r.each = __builtin_amdgcn_readfirstlane(r.each);
}
// Leaves where the parts of an output are: first worker, parts (0: it is whole), and
// which of its first worker's parts is the first.
__device__ __forceinline__ void note_parts(const TreeArg& a, const TreeRun& r, int w, int hk, int units, int s1,
                                           bool first_segment) {
  int32_t* h = a.heads_of + 3 * (((int64_t)r.tr * a.blocks + r.cb) * a.kv.n_kv_heads + hk);
  h[0] = w;
  h[1] = s1 == units ? 0 : r.each ? (units + r.each - 1) / r.each : (r.base + units - 1) / r.run - w + 1;
  h[2] = first_segment ? 0 : 1;
}

// A column is a query head of a key head's group, of one node: column c is node
// c / group, head c % group.  A workgroup takes a block of 16 * kTiles columns of a
// tree and a run of its keys, each wavefront every fourth tile of 32 keys, for all
// columns of the block; statistics and outputs of a column stay in the lanes of its
// own (Tile says how).  The softmax runs once over the keys with a running maximum.
//
// Outputs that a worker covers whole it writes; of the others (its first and its last at
// most) it leaves maximum, sum and unscaled output in the workspace, which
// tree_join_kernel joins.
//
// A tile that all columns see whole has nothing masked.  In the others (the tree's
// own keys, the window's edge, missing pages) a weight of 0 would not undo an
// infinity or a NaN among the values, which the columns share: keys with such
// values are cleared from the product and added by themselves, to the columns that
// see them.
//
// Bound by HBM where there are keys enough: 64 trees of one node and 1,001 keys of 8 heads of
// 128 take 46 us, 5.7 TB/s.  Short calls are bound by the chain of trips to memory (lengths,
// page table, keys, values) and two launches.  With four tiles of columns, 64 to a wavefront,
// registers ran out: 40 trees over 8 bits 389 us, which the wide kernel takes in 160.
template <class T, bool kE4M3, int kDh, int kTiles, bool kShaped>
__global__ __launch_bounds__(64 * kTreeWaves, kDh == 256 ? 1 : 2)
void paged_tree_kernel(TreeArg a) {
  constexpr int kWaves = kTreeWaves, kThreads = 64 * kWaves, kColumns = 16 * kTiles;
  typedef WideTile<T, kE4M3, kDh, kTiles> Tl;
  constexpr int kRow = kDh + 4;  // padded: lanes 16 apart in dimensions, 1 in columns
  __shared__ float ms[kWaves][kColumns], ls[kWaves][kColumns];
  __shared__ __attribute__((aligned(16))) float os[kWaves][16][kRow];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g4 = lane >> 4;
  const uint32_t k_off = Tl::k_offset(lane, a.kv.slot_bytes);
  const uint32_t v_off = Tl::v_offset(lane, a.kv.slot_bytes);

  // Workgroups of several key heads stand next to each other, as their keys do in memory.
  const int hk = blockIdx.x, w = a.workers ? blockIdx.y : blockIdx.z, cb = a.workers ? 0 : blockIdx.y;
  TreeChunk ch;
  TreeRun r{0, 1, 0, w, cb, 1, 0};
  if (a.workers) {
    if (!find_run(a, w, kColumns, ch, r)) return;  // the same for the whole workgroup
  } else {
    ch.load(a, w & ~63, kColumns);
    if (cb >= __builtin_amdgcn_readlane(ch.blocks, w & 63)) return;
  }

  float scale = a.scale;
  if (!kShaped) scale *= 1.4426950408889634f;
  if (kE4M3 && a.kv.k_scale) scale *= a.kv.k_scale[hk];
  const uint32_t flip = scale < 0.f ? 0x80008000u : 0u;
  scale = fabsf(scale);
  const float vs = kE4M3 && a.kv.v_scale ? a.kv.v_scale[hk] : 1.f;
  const float inv_cap = kShaped && a.cap > 0.f ? 1.f / a.cap : 0.f;
  const uint8_t* kbase = a.kv.k + (int64_t)hk * a.kv.head_bytes;
  const uint8_t* vbase = a.kv.v + (int64_t)hk * a.kv.head_bytes;
  const int slot_mask = (1 << a.kv.page_log2) - 1;
  bool first_segment = true;

  make_uniform(r);
  while (r.u < r.u_end) {
    make_uniform(r);
    if (r.tr - ch.first >= 64) ch.load(a, r.tr & ~63, kColumns);
    const int i64 = __builtin_amdgcn_readfirstlane(r.tr - ch.first);
    if (r.cb >= __builtin_amdgcn_readlane(ch.blocks, i64)) {
      r.cb = 0;
      ++r.tr;
      continue;
    }
    const int start = __builtin_amdgcn_readlane(ch.span.start, i64);
    const int count = __builtin_amdgcn_readlane(ch.span.count, i64);
    const int sq = __builtin_amdgcn_readlane(ch.span.seq, i64);
    const int n = __builtin_amdgcn_readlane(ch.span.n, i64);
    const int first = __builtin_amdgcn_readlane(ch.span.first, i64);
    const int end = __builtin_amdgcn_readlane(ch.span.end, i64);
    const int units = a.workers ? __builtin_amdgcn_readlane(ch.units, i64) : 1;
    const int s0 = r.u - r.base, s1 = min(units, s0 + (r.u_end - r.u));
    const int columns = min(kColumns, count * a.group - r.cb * kColumns);

    // This lane's columns: node, and what belongs to it.
    int node[kTiles];
    float slope[kTiles];
    int deep_at[kTiles];
    uint4 q[kTiles][Tl::kSteps];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int c = 16 * i + l16, col = r.cb * kColumns + c;
      node[i] = c < columns ? (int)((uint32_t)col / (uint32_t)a.group) : 0;
      const int head = hk * a.group + (c < columns ? col - node[i] * a.group : 0);
      slope[i] = 0.f;
      if (kShaped && a.slopes) slope[i] = a.slopes[head] * 1.4426950408889634f;
#pragma unroll
      for (int s = 0; s < Tl::kSteps; ++s) {
        q[i][s] = make_uint4(0, 0, 0, 0);
        if (c < columns)
          q[i][s] = signed_chunk(a.q + (int64_t)(start + node[i]) * a.q_stride + (int64_t)head * kDh + Tl::q_dim(s, g4),
                                 flip);
      }
    }
    f32x4 acc[kTiles][Tl::kDims];
    float m[kTiles], l[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < Tl::kDims; ++c) acc[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const int t0 = first / kTileKeys, t_all = (end + kTileKeys - 1) / kTileKeys;
    const int t_end = a.workers ? min(t0 + s1 * kWaves, t_all) : t_all;
    int t = t0 + s0 * kWaves + wave;
    const ConstI32 table = (ConstI32)(a.table + (int64_t)sq * a.table_stride);

    auto place = [&](const Octets& o, int key0, int64_t (&off)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int page = (uint32_t)o.page[i] < (uint32_t)a.kv.n_pages ? o.page[i] : 0;
        off[i] = page * a.kv.page_bytes + (int64_t)((key0 + 8 * i) & slot_mask) * a.kv.slot_bytes;
      }
    };
    Tl tile;
    auto load_k = [&](const int64_t (&off)[4]) {
      const uint8_t* const p[4] = {kbase + off[0], kbase + off[1], kbase + off[2], kbase + off[3]};
      tile.load_k(p, k_off);
    };
    auto load_v = [&](const int64_t (&off)[4]) {
      const uint8_t* const p[4] = {vbase + off[0], vbase + off[1], vbase + off[2], vbase + off[3]};
      tile.load_v(p, a.kv.slot_bytes, v_off);
    };

    Octets now, next;
    int64_t off[4];
    if (t < t_end) {
      now = octets_of(a.kv, table, t * kTileKeys, end);
      place(now, t * kTileKeys, off);
      load_k(off);
      load_v(off);
      if (t + kWaves < t_end) next = octets_of(a.kv, table, (t + kWaves) * kTileKeys, end);
    }
    // What each node sees, and its depth: node i's in lane i.
    uint64_t sees = 0;
    if (lane < count)
      sees = a.tree ? a.tree[start + lane] : (2ull << lane) - 1;
    const int depth = __popcll(sees & ((1ull << lane) - 1));
    const int deepest = a.window > 0 ? (int)wave_reduce_u32<true>((uint32_t)(lane < count ? depth : 0)) : 0;

#pragma unroll
    for (int i = 0; i < kTiles; ++i) deep_at[i] = kShaped ? __shfl(depth, node[i]) : 0;
    // Keys of a tile that every column sees lie between these.
    const int low = a.window > 0 ? max(0, n + deepest + 1 - a.window) : 0, high = min(n, end);
    while (t < t_end) {
      const int key0 = t * kTileKeys, tn = t + kWaves;
      const bool more = tn < t_end;
      f32x4 s[kTiles][2];
      tile.wide_scores(q, (lane & 2) != 0, s);
      if (more) {
        place(next, tn * kTileKeys, off);
        load_k(off);
      }
      bool whole = key0 >= low && key0 + kTileKeys <= high;
#pragma unroll
      for (int i = 0; i < 4; ++i) whole = whole && (uint32_t)now.page[i] < (uint32_t)a.kv.n_pages;
      auto key_of = [&](int j, int group) { return key0 + 8 * (j >> 1) + 2 * group + (j & 1); };
      float z[kTiles][8];
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[i][j] = kShaped ? s[i][j >> 2][j & 3] * scale : s[i][j >> 2][j & 3];
      if constexpr (kShaped) {
        int key_at[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) key_at[j] = key_of(j, g4) - n;
        shape_scores(z, a.cap, inv_cap, a.slopes != nullptr, slope, deep_at, key_at, key0 + kTileKeys > n, depth);
      }
      uint32_t bad = 0, seen[kTiles];
      if (!whole) {
        uint32_t octets = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) octets |= (uint32_t)now.page[i] < (uint32_t)a.kv.n_pages ? 1u << i : 0u;
        const uint32_t there = keys_there(key0, first, end, octets), own = there >> (2 * g4);
        uint32_t keep = 0;  // a bit for each of the lane's keys
#pragma unroll
        for (int j = 0; j < 8; ++j) keep |= (own >> (8 * (j >> 1) + (j & 1)) & 1) << j;
        tile.clear_v(keep);
        if (__builtin_expect(__any(tile.any_not_finite()), 0)) {
          bad = tile.not_finite();
          bad |= __shfl_xor(bad, 1);
          bad |= __shfl_xor(bad, 2);
          bad |= __shfl_xor(bad, 4);
          bad |= __shfl_xor(bad, 8);
        }
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          seen[i] = there & keys_seen(key0, n, __shfl(sees, node[i]), __shfl(depth, node[i]), a.window, depth);
          const uint32_t mine = seen[i] >> (2 * g4);
#pragma unroll
          for (int j = 0; j < 8; ++j) z[i][j] = mine >> (8 * (j >> 1) + (j & 1)) & 1 ? z[i][j] : -INFINITY;
        }
      }
      float p[kTiles][8];
      soft_step<Tl>(z, kShaped ? 1.f : scale, !whole, m, l, acc, p);
      if (__builtin_expect(__any(bad != 0), 0)) {
#pragma unroll 1
        for (int x = 0; x < 32; ++x) {
          const int j = x & 7, kg = x >> 3;
          if (!((__builtin_amdgcn_readlane((int)bad, 16 * kg) >> j) & 1)) continue;
          const int at = 8 * (j >> 1) + 2 * kg + (j & 1);
          float weight[kTiles];
          bool sees_it[kTiles];
#pragma unroll
          for (int i = 0; i < kTiles; ++i) {
            weight[i] = weight_of(p[i], j, kg);
            sees_it[i] = seen[i] >> at & 1;
          }
          tile.template add_key<0>(j, g4 == kg, weight, sees_it, acc);
        }
        tile.clear_v(~bad);
      }
      bool again = false;
      add_in_halves<Tl>(p, acc, [&](const uint4(&hi)[kTiles][1], const uint4(&lo)[kTiles][1]) __attribute__((always_inline)) {
        if (again) tile.transpose_again();
        again = true;
        tile.template wide_add<0>(hi, lo, acc);
      });
      if (more) {
        load_v(off);
        now = next;
        if (tn + kWaves < t_end) next = octets_of(a.kv, table, (tn + kWaves) * kTileKeys, end);
      }
      t = tn;
    }

    // Join the wavefronts, a tile of columns at a time.
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      l[i] += __shfl_xor(l[i], 16);
      l[i] += __shfl_xor(l[i], 32);
    }
    __syncthreads();  // the last segment's readers are done
    if (g4 == 0) {
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        ms[wave][16 * i + l16] = m[i];
        ls[wave][16 * i + l16] = l[i];
      }
    }
    __syncthreads();
    const bool full = s0 == 0 && s1 == units;
    float* part = a.parts + (int64_t)(2 * (w * a.kv.n_kv_heads + hk) + (first_segment ? 0 : 1)) * a.part_floats;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      if (16 * i >= columns) break;
      if (i > 0) __syncthreads();
      float M = ms[0][16 * i + l16];
#pragma unroll
      for (int v = 1; v < kWaves; ++v) M = fmaxf(M, ms[v][16 * i + l16]);
      const float f = part_weight(m[i], M);
#pragma unroll
      for (int c = 0; c < Tl::kDims; c += 4)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<float4*>(&os[wave][l16][Tl::out_dim(4 * g4 + q4, c)]) =
              make_float4(acc[i][c][q4] * f, acc[i][c + 1][q4] * f, acc[i][c + 2][q4] * f, acc[i][c + 3][q4] * f);
      __syncthreads();
      for (int x = tid; x < min(16, columns - 16 * i) * (kDh / 4); x += kThreads) {
        const int h = x / (kDh / 4), d = 4 * (x % (kDh / 4)), c = 16 * i + h;
        float4 o = *reinterpret_cast<const float4*>(&os[0][h][d]);
#pragma unroll
        for (int v = 1; v < kWaves; ++v) {
          const float4 e = *reinterpret_cast<const float4*>(&os[v][h][d]);
          o.x += e.x, o.y += e.y, o.z += e.z, o.w += e.w;
        }
        float top = ms[0][c], sum = 0.f;
#pragma unroll
        for (int v = 1; v < kWaves; ++v) top = fmaxf(top, ms[v][c]);
#pragma unroll
        for (int v = 0; v < kWaves; ++v) sum += ls[v][c] * part_weight(ms[v][c], top);
        if (full) {
          const int col = r.cb * kColumns + c, nd = (int)((uint32_t)col / (uint32_t)a.group);
          const int64_t row = start + nd;
          const int head = hk * a.group + col - nd * a.group;
          const float inv = sum == 0.f ? 0.f : vs / sum;
          uint2 four;
          four.x = T::down(o.x * inv) | (T::down(o.y * inv) << 16);
          four.y = T::down(o.z * inv) | (T::down(o.w * inv) << 16);
          *reinterpret_cast<uint2*>(a.out + row * a.out_stride + (int64_t)head * kDh + d) = four;
          if (d == 0 && a.lse)
            a.lse[row * a.n_heads + head] =
                sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
        } else {
          *reinterpret_cast<float4*>(part + 2 * kColumns + c * kDh + d) = o;
          if (d == 0) {
            part[c] = top;
            part[kColumns + c] = sum;
          }
        }
      }
    }
    if (a.workers && s0 == 0 && tid == 0) note_parts(a, r, w, hk, units, s1, first_segment);
    r.u += s1 - s0;
    r.base += units;
    ++r.cb;
    first_segment = false;
  }
}

// Joins the parts of an output that workers shared, kStripes threads to four dimensions of a
// column, each over every kStripes-th part: weights of a part are 2^(its maximum - the
// largest).  Reads 4 bytes a column, dimension and part, and writes the output; its time is
// its launch and the chain descriptors, maxima, parts, about 4 us of the smallest calls.
template <class T, bool kE4M3, int kDh, int kStripes>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArg a, int tiles) {
  __shared__ float4 so[256];
  __shared__ float sm[256], sl[256];
  constexpr int kItems = 256 / kStripes, kFours = kDh / 4;
  const int columns = 16 * tiles, pieces = columns * kFours / kItems;
  const int output = blockIdx.x / pieces, piece = blockIdx.x % pieces;
  const int hk = output % a.kv.n_kv_heads, cb = output / a.kv.n_kv_heads % a.blocks;
  const int tr = output / a.kv.n_kv_heads / a.blocks;
  const TreeSpan s = tree_span(a, a.tree0 + tr);
  if (s.count * a.group <= cb * columns) return;
  const int32_t* h = a.heads_of + 3 * (int64_t)output;
  const int w = h[0], parts = h[1], lead = h[2];
  if (parts == 0) return;
  const int item = piece * kItems + threadIdx.x % kItems, stripe = threadIdx.x / kItems;
  const int c = item / kFours, d = 4 * (item % kFours), col = cb * columns + c;
  float M = -INFINITY, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kAhead = kStripes == 1 ? 8 : 4;  // parts under way (328 keys in 6 parts: 13.0 us with 8, 12.6 with 4)
  if (col < s.count * a.group) {
    for (int i0 = stripe; i0 < parts; i0 += kAhead * kStripes) {
      float m_of[kAhead], l_of[kAhead];
      float4 e[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = min(i0 + k * kStripes, parts - 1);
        const float* p = a.parts + (2 * ((int64_t)(w + i) * a.kv.n_kv_heads + hk) + (i == 0 ? lead : 0)) * a.part_floats;
        m_of[k] = p[c];
        l_of[k] = p[columns + c];
        e[k] = *reinterpret_cast<const float4*>(p + 2 * columns + c * kDh + d);
      }
      float top = M;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (i0 + k * kStripes >= parts) {  // past the end: nothing (an infinity times 0 is not)
          m_of[k] = -INFINITY;
          l_of[k] = 0.f;
          e[k] = make_float4(0.f, 0.f, 0.f, 0.f);
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
        o.x = fmaf(f, e[k].x, o.x), o.y = fmaf(f, e[k].y, o.y);
        o.z = fmaf(f, e[k].z, o.z), o.w = fmaf(f, e[k].w, o.w);
      }
    }
  }
  if constexpr (kStripes > 1) {
    so[threadIdx.x] = o;
    sm[threadIdx.x] = M;
    sl[threadIdx.x] = L;
    __syncthreads();
    if (stripe != 0) return;
    M = sm[threadIdx.x];
    for (int i = 1; i < kStripes; ++i) M = fmaxf(M, sm[threadIdx.x + i * kItems]);
    L = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < kStripes; ++i) {
      const int x = threadIdx.x + i * kItems;
      const float f = part_weight(sm[x], M);
      L = fmaf(f, sl[x], L);
      o.x = fmaf(f, so[x].x, o.x), o.y = fmaf(f, so[x].y, o.y);
      o.z = fmaf(f, so[x].z, o.z), o.w = fmaf(f, so[x].w, o.w);
    }
  }
  if (col >= s.count * a.group) return;
  const int nd = (int)((uint32_t)col / (uint32_t)a.group), head = hk * a.group + col - nd * a.group;
  const int64_t row = s.start + nd;
  const float vs = kE4M3 && a.kv.v_scale ? a.kv.v_scale[hk] : 1.f, inv = L == 0.f ? 0.f : vs / L;
  uint2 r;
  r.x = T::down(o.x * inv) | (T::down(o.y * inv) << 16);
  r.y = T::down(o.z * inv) | (T::down(o.w * inv) << 16);
  *reinterpret_cast<uint2*>(a.out + row * a.out_stride + (int64_t)head * kDh + d) = r;
  if (d == 0 && a.lse)
    a.lse[row * a.n_heads + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

}  // namespace emoe
