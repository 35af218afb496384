// The tree attention's kernel for many columns (exactmoe_drafts.h): wavefronts share
// the keys and take columns of their own.
#pragma once

#include "tree.h"

namespace emoe {

// Wait until at most kLeft of this wavefront's loads are under way.
template <int kLeft>
__device__ __forceinline__ void wait_loads() {
  static_assert(kLeft < 64, "vmcnt");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((kLeft & 15) | ((kLeft >> 4) << 14) | (0x7 << 4) | (0xF << 8));
  asm volatile("" ::: "memory");
}
// Workgroup barrier that orders LDS accesses but does not wait for loads.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xF | (0x3 << 14) | (0x7 << 4));  // lgkmcnt(0) only
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Copies 16 bytes per lane, from `from` + offset, to LDS, at `to` + 16 * lane, past the
// caches (131,072 keys: 122 -> 104 us).  As assembly, since the compiler would have every
// read of LDS wait for all copies under way; it has no registers as outputs, and the
// kernel itself waits for it.  M0, which it changes, is named, so that the compiler does not
// take a value that it put there before for still there after; that it is none of those
// that the compiler would save is what the warning says.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(const uint8_t* from, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(
                   __builtin_amdgcn_readfirstlane(to)),
               "v"(offset), "s"(from)
               : "memory", "m0");
}
__device__ __forceinline__ void copy_to_lds(const uint8_t* from, uint32_t to) {  // from: of each lane
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(
                   __builtin_amdgcn_readfirstlane(to)),
               "v"(from)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// A ring of tiles of 32 keys and their values in LDS.  Row r of a tile holds its 16-byte
// chunks in the order c ^ swizzle(r) (values: swizzle_v), so that lanes that read the same
// chunk of several rows use all banks.  The kernel takes steps of one or two tiles, and
// as many as the LDS of a workgroup's share of a CU holds, up to four, are under way.
template <int kDh, bool kE4M3>
struct WideRing {
  static constexpr int kRow = kDh * (kE4M3 ? 1 : 2), kSide = 32 * kRow, kTile = 2 * kSide;
  static constexpr int kStepTiles = wide_step_tiles(kDh, kE4M3), kStep = kStepTiles * kTile;
  static constexpr int kFit = 160 * 1024 / wide_workgroups(kDh, kE4M3) / (kStep + 64);
  static constexpr int kSteps = kFit < 4 ? kFit : 4;
  static constexpr int kCopies = kStep / 4096;  // of a wavefront and step

  __device__ static __forceinline__ int swizzle(int row) { return kRow == 64 ? (row >> 1) & 3 : row & 7; }
  // Of values, which are read transposed: 4 rows of 32 bytes at once, or 8 of 16 (8 bits).
  __device__ static __forceinline__ int swizzle_v(int row) {
    return !kE4M3 ? 2 * (row & 3) : kRow == 64 ? (row >> 1 & 1) | (row >> 3 & 2) : (row & 3) | (row >> 2 & 4);
  }
  __device__ static __forceinline__ uint8_t* memory() {
    __shared__ __attribute__((aligned(1024))) uint8_t ring[kSteps * kStep];
    return ring;
  }
  // Of each step and wavefront, whether all octets that it copies are there.
  __device__ static __forceinline__ uint32_t (*whole())[4] {
    __shared__ __attribute__((aligned(16))) uint32_t words[kSteps][4];
    return words;
  }
};

// One block of 64 columns of a tree over a run of its keys, 16 columns to a wavefront.
template <class T, bool kE4M3, int kDh, bool kShaped>
struct WideSegment {
  static constexpr int kTiles = 1;  // of 16 columns, of a wavefront
  static constexpr int kColumns = 64 * kTiles;
  typedef WideTile<T, kE4M3, kDh, kTiles> Tl;
  typedef WideRing<kDh, kE4M3> Ring;
  static constexpr int kRow = Ring::kRow, kItem = Tl::kItem;
  static constexpr int kSub = kE4M3 ? 2 : 1;         // steps of a 16-byte chunk of keys
  static constexpr int kChunks = kRow / 64;          // chunks of a lane
  // Tiles of 32 keys of a step, which are taken together (more to do while a product or a
  // read is under way), and a lane's keys of them.
  static constexpr int kU = Ring::kStepTiles, kKeys = 8 * kU;
  static constexpr int kBlocks = kDh / 16;            // of output dimensions

  // The halves of these values whose exponent is of ones only (infinities and NaN): each
  // one's highest bit.
  __device__ static __forceinline__ uint4 not_finite(const uint4& v) {
    constexpr uint32_t kOne = Tl::kF16Weights ? 0x04000400u : 0x00800080u, kAbs = 0x7fff7fffu;
    return make_uint4((v.x & kAbs) + kOne, (v.y & kAbs) + kOne, (v.z & kAbs) + kOne, (v.w & kAbs) + kOne);
  }
  // The values of the keys that are not in `keep` become 0.
  __device__ static __forceinline__ uint4 cleared_values(const uint4& v, uint32_t keep) {
    uint32_t m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      m[i] = ((keep >> (2 * i)) & 1 ? 0xffffu : 0u) | ((keep >> (2 * i)) & 2 ? 0xffff0000u : 0u);
    return make_uint4(v.x & m[0], v.y & m[1], v.z & m[2], v.w & m[3]);
  }

  // Dimension of the first element that lane group g has of step s.
  __device__ static __forceinline__ int q_dim(int s, int g) {
    return (16 / kItem) * (4 * (s / kSub) + g) + 8 * (s % kSub);
  }

  // Copies the wavefront's octet of a tile, which is in `page`.
  __device__ static __forceinline__ void fetch(const TreeArg& a, uint32_t tile_at, const uint8_t* kbase,
                                               const uint8_t* vbase, int key0, int page, int wave, int lane) {
    constexpr int kRowsAtOnce = 1024 / kRow;
    const int64_t at = ((uint32_t)page < (uint32_t)a.kv.n_pages ? page : 0) * a.kv.page_bytes +
                       (int64_t)((key0 + 8 * wave) & ((1 << a.kv.page_log2) - 1)) * a.kv.slot_bytes;
    if constexpr (kRowsAtOnce == 16) {  // keys from the lower half of the lanes, values from the upper one
      const int row = (lane >> 2) & 7;
      const int swizzle = lane < 32 ? Ring::swizzle(row) : Ring::swizzle_v(8 * wave + row);
      const uint8_t* from = (lane < 32 ? kbase : vbase) + at + (uint32_t)(row * a.kv.slot_bytes) +
                            16 * ((lane & 3) ^ swizzle);
      copy_to_lds(from, tile_at + 1024 * wave);
    } else {
      const int in = lane / (kRow / 16), chunk = lane % (kRow / 16);
#pragma unroll
      for (int i = 0; i < 8 / kRowsAtOnce; ++i) {
        const int row = i * kRowsAtOnce + in;
        const uint32_t slot = row * a.kv.slot_bytes;
        const uint32_t to = tile_at + (8 * wave + i * kRowsAtOnce) * kRow;
        copy_to_lds(kbase + at, slot + 16 * (chunk ^ Ring::swizzle(row)), to);
        copy_to_lds(vbase + at, slot + 16 * (chunk ^ Ring::swizzle_v(8 * wave + row)), to + Ring::kSide);
      }
    }
  }
  // Where a row's keys and values are in a tile.
  static constexpr bool kMixed = kRow == 64;  // octets of keys and of values in turn
  __device__ static __forceinline__ int key_row(int row) { return kMixed ? 1024 * (row >> 3) + 64 * (row & 7) : row * kRow; }
  static constexpr int kValues = kMixed ? 512 : Ring::kSide;

  __device__ static __forceinline__ void run(const TreeArg& a, const TreeRun& r, int w, int hk, int start,
                                             int count, int sq, int n, int first, int end, int units, int s0,
                                             int s1, int columns, bool first_segment) {
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g4 = lane >> 4;
    const bool active = 16 * wave < columns;

    float scale = a.scale;
    if (!kShaped) scale *= 1.4426950408889634f;
    if (kE4M3 && a.kv.k_scale) scale *= a.kv.k_scale[hk];
    const uint32_t flip = scale < 0.f ? 0x80008000u : 0u;
    scale = fabsf(scale);
    const float inv_cap = kShaped && a.cap > 0.f ? 1.f / a.cap : 0.f;
    const uint8_t* kbase = a.kv.k + (int64_t)hk * a.kv.head_bytes;
    const uint8_t* vbase = a.kv.v + (int64_t)hk * a.kv.head_bytes;
    const ConstI32 table = (ConstI32)(a.table + (int64_t)sq * a.table_stride);

    constexpr int kStepKeys = 32 * kU, kAhead = Ring::kSteps - 1;
    const int t_all = (end + kStepKeys - 1) / kStepKeys, t0 = first / kStepKeys;
    int t = t0 + s0;
    const int t_end = a.workers ? min(t0 + s1, t_all) : t_all;
    uint8_t* ring = Ring::memory();
    const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)ring;
    auto page_of = [&](int key) -> int { return key < end ? table[key >> a.kv.page_log2] : -1; };
    struct Pages {
      int32_t tile[kU];
    };
    auto pages_of = [&](int step) -> Pages {  // of the octets that this wavefront copies
      Pages o;
#pragma unroll
      for (int u = 0; u < kU; ++u) o.tile[u] = page_of(step * kStepKeys + 32 * u + 8 * wave);
      return o;
    };
    auto fetch_step = [&](int step, const Pages& o) {
      bool all = true;
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        all = all && (uint32_t)o.tile[u] < (uint32_t)a.kv.n_pages;
        fetch(a, ring_at + (step % Ring::kSteps) * Ring::kStep + u * Ring::kTile, kbase, vbase,
              step * kStepKeys + 32 * u, o.tile[u], wave, lane);
      }
      if (lane == 0) Ring::whole()[step % Ring::kSteps][wave] = all ? 1u : 0u;
    };
    lds_barrier();  // the last segment's readers are done
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (t + i < t_end) {
        const Pages o = pages_of(t + i);
        fetch_step(t + i, o);
      }
    }
    // What each node sees, and its depth: node i's in lane i.
    uint64_t sees = 0;
    if (lane < count) sees = a.tree ? a.tree[start + lane] : (2ull << lane) - 1;
    const int depth = __popcll(sees & ((1ull << lane) - 1));
    const int deepest = a.window > 0 ? (int)wave_reduce_u32<true>((uint32_t)(lane < count ? depth : 0)) : 0;
    int node[kTiles], deep_at[kTiles];
    float slope[kTiles];
    uint4 q[kTiles][Tl::kSteps];
    f32x4 acc[kTiles][kBlocks];
    float m[kTiles], l[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int c = 16 * wave + l16, col = r.cb * kColumns + c;
      node[i] = c < columns ? (int)((uint32_t)col / (uint32_t)a.group) : 0;
      const int head = hk * a.group + (c < columns ? col - node[i] * a.group : 0);
      slope[i] = 0.f;
      deep_at[i] = kShaped ? __shfl(depth, node[i]) : 0;
      if (kShaped && a.slopes) slope[i] = a.slopes[head] * 1.4426950408889634f;
#pragma unroll
      for (int s = 0; s < Tl::kSteps; ++s) {
        q[i][s] = make_uint4(0, 0, 0, 0);
        if (c < columns)
          q[i][s] = signed_chunk(a.q + (int64_t)(start + node[i]) * a.q_stride + (int64_t)head * kDh + q_dim(s, g4), flip);
      }
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < kBlocks; ++c) acc[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int low = a.window > 0 ? max(0, n + deepest + 1 - a.window) : 0, high = min(n, end);
    // A lane's places in a tile: its keys' chunks (even and odd), its part of the values.
    int k_at[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      k_at[i] = key_row(l16) + 16 * ((g4 | (kRow == 64 ? 0 : 4 * i)) ^ Ring::swizzle(l16));
    // 16 bits: row 4 g4 + l16 / 4, 8 bytes l16 % 4 of 32; 8 bits: row r = l16 / 2 of the
    // group's eight, 8 bytes l16 % 2 of 16.
    const int v_row = kE4M3 ? 4 * g4 + (l16 >> 1 & 3) + 16 * (l16 >> 3) : 4 * g4 + (l16 >> 2);
    const int v_at = kValues + key_row(v_row) + 8 * (l16 & 1);
    const int v_swizzle = Ring::swizzle_v(v_row);
    constexpr int kHalf = kMixed ? 2048 : 16 * kRow;  // from row r to row r + 16

    auto compute = [&](const uint8_t* held, int key0, bool all) __attribute__((always_inline)) {
      f32x4 s[kTiles][2 * kU];
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int h = 0; h < 2 * kU; ++h) s[i][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = 0; p < kChunks; ++p)
#pragma unroll
        for (int h = 0; h < 2 * kU; ++h) {
          const uint4 c = *reinterpret_cast<const uint4*>(held + k_at[p & 1] + (h >> 1) * Ring::kTile +
                                                          (h & 1) * kHalf + 128 * (p >> 1));
          if constexpr (kE4M3) {
            typedef typename Tl::H16 H;
            const uint4 x0 = make_uint4(H::template from_e4m3<false>(c.x), H::template from_e4m3<true>(c.x),
                                        H::template from_e4m3<false>(c.y), H::template from_e4m3<true>(c.y));
            const uint4 x1 = make_uint4(H::template from_e4m3<false>(c.z), H::template from_e4m3<true>(c.z),
                                        H::template from_e4m3<false>(c.w), H::template from_e4m3<true>(c.w));
#pragma unroll
            for (int i = 0; i < kTiles; ++i) s[i][h] = H::mfma(x0, q[i][2 * p], s[i][h]);
#pragma unroll
            for (int i = 0; i < kTiles; ++i) s[i][h] = H::mfma(x1, q[i][2 * p + 1], s[i][h]);
          } else {
#pragma unroll
            for (int i = 0; i < kTiles; ++i) s[i][h] = Tl::H16::mfma(c, q[i][p], s[i][h]);
          }
        }
      // The values of dimensions 16 c + l16 of the lane group's 8 keys of a tile, in the
      // order of the scores: LDS transposes them on the way.
      auto values = [&](int c, int u) __attribute__((always_inline)) -> uint4 {
        const uint8_t* tile = held + u * Ring::kTile;
        if constexpr (kE4M3) {
          typedef int i32x2 __attribute__((ext_vector_type(2)));
          typedef __attribute__((address_space(3))) i32x2* At;
          const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((At)(tile + v_at + 16 * (c ^ v_swizzle)));
          return make_uint4(Tl::HW::template from_e4m3<false>((uint32_t)x[0]),
                            Tl::HW::template from_e4m3<true>((uint32_t)x[0]),
                            Tl::HW::template from_e4m3<false>((uint32_t)x[1]),
                            Tl::HW::template from_e4m3<true>((uint32_t)x[1]));
        } else {
          typedef short i16x4 __attribute__((ext_vector_type(4)));
          typedef __attribute__((address_space(3))) i16x4* At;
          const uint8_t* at = tile + v_at + 16 * ((2 * c + (l16 >> 1 & 1)) ^ v_swizzle);
          const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)at));
          const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(at + kHalf)));
          return make_uint4(x.x, x.y, y.x, y.y);
        }
      };
      // The place in the step of a lane group's key j, and its octet.
      auto key_of = [&](int j, int group) { return 32 * (j >> 3) + 16 * (j >> 2 & 1) + 4 * group + (j & 3); };
      float z[kTiles][kKeys], p[kTiles][kKeys];
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int j = 0; j < kKeys; ++j) z[i][j] = kShaped ? s[i][j >> 2][j & 3] * scale : s[i][j >> 2][j & 3];
      if constexpr (kShaped) {
        int key_at[kKeys];
#pragma unroll
        for (int j = 0; j < kKeys; ++j) key_at[j] = key0 + key_of(j, g4) - n;
        shape_scores(z, a.cap, inv_cap, a.slopes != nullptr, slope, deep_at, key_at, key0 + 32 * kU > n, depth);
      }
      uint32_t bad = 0, keep = ~0u;
      uint32_t seen[kTiles] = {}, seen_next[kTiles] = {};  // keys of the first and of the second tile
      const bool masked = !(key0 >= low && key0 + 32 * kU <= high && all);
      if (masked) {
        keep = 0;
        uint32_t any = 0;
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          uint32_t octets = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            octets |= (uint32_t)page_of(key0 + 32 * u + 8 * i) < (uint32_t)a.kv.n_pages ? 1u << i : 0u;
          const uint32_t there = keys_there(key0 + 32 * u, first, end, octets);
          const uint32_t own = there >> (4 * g4);
          keep |= ((own & 15) | (own >> 12 & 0xf0)) << (8 * u);
#pragma unroll
          for (int c = 0; c < kBlocks; ++c) {
            const uint4 x = not_finite(cleared_values(values(c, u), keep >> (8 * u)));
            any |= x.x | x.y | x.z | x.w;
          }
#pragma unroll
          for (int i = 0; i < kTiles; ++i) {
            const uint32_t bits =
                there & keys_seen(key0 + 32 * u, n, __shfl(sees, node[i]), __shfl(depth, node[i]), a.window, depth);
            if (u == 0) seen[i] = bits;
            else seen_next[i] = bits;
            const uint32_t mine = bits >> (4 * g4);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              z[i][8 * u + j] = mine >> (16 * (j >> 2) + (j & 3)) & 1 ? z[i][8 * u + j] : -INFINITY;
          }
        }
        if (__builtin_expect(__any((any & 0x80008000u) != 0), 0)) {
#pragma unroll
          for (int u = 0; u < kU; ++u)
#pragma unroll 1
            for (int c = 0; c < kBlocks; ++c) {
              const uint4 x = not_finite(cleared_values(values(c, u), keep >> (8 * u)));
              const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
              for (int j = 0; j < 8; ++j) bad |= (w[j >> 1] >> (16 * (j & 1) + 15) & 1) << (8 * u + j);
            }
          bad |= __shfl_xor(bad, 1);
          bad |= __shfl_xor(bad, 2);
          bad |= __shfl_xor(bad, 4);
          bad |= __shfl_xor(bad, 8);
          keep &= ~bad;
        }
      }
      soft_step<Tl>(z, kShaped ? 1.f : scale, masked, m, l, acc, p);
      if (__builtin_expect(__any(bad != 0), 0)) {
#pragma unroll 1
        for (int x = 0; x < 4 * kKeys; ++x) {
          const int j = x % kKeys, kg = x / kKeys, at = key_of(j, kg);
          if (!((__builtin_amdgcn_readlane((int)bad, 16 * kg) >> j) & 1)) continue;
          float weight[kTiles];
          bool sees_it[kTiles];
#pragma unroll
          for (int i = 0; i < kTiles; ++i) {
            weight[i] = weight_of(p[i], j, kg);
            sees_it[i] = (((uint64_t)seen_next[i] << 32 | seen[i]) >> at) & 1;
          }
          const uint32_t only = g4 == kg ? 1u << (j & 7) : 0u;
          constexpr uint32_t kOne = Tl::kF16Weights ? 0x3c003c00u : 0x3f803f80u;
          const uint4 one = cleared_values(make_uint4(kOne, kOne, kOne, kOne), only);
#pragma unroll
          for (int c = 0; c < kBlocks; ++c) {  // a weight of 1 brings its values to the output's lanes
            const f32x4 v = Tl::HW::mfma(cleared_values(values(c, j >> 3), only), one, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int i = 0; i < kTiles; ++i) acc[i][c] = add_where(sees_it[i], weight[i], v, acc[i][c]);
          }
        }
      }
      add_in_halves<Tl>(p, acc, [&](const uint4(&hi)[kTiles][kU], const uint4(&lo)[kTiles][kU])
                                    __attribute__((always_inline)) {
        auto add = [&](auto cleared) __attribute__((always_inline)) {
#pragma unroll
          for (int c = 0; c < kBlocks; ++c)
#pragma unroll
            for (int u = 0; u < kU; ++u) {
              uint4 v = values(c, u);
              if constexpr (decltype(cleared)::value) v = cleared_values(v, keep >> (8 * u));
#pragma unroll
              for (int i = 0; i < kTiles; ++i) acc[i][c] = Tl::HW::mfma(v, hi[i][u], acc[i][c]);
#pragma unroll
              for (int i = 0; i < kTiles; ++i) acc[i][c] = Tl::HW::mfma(v, lo[i][u], acc[i][c]);
            }
        };
        if (masked) add(std::true_type());
        else add(std::false_type());
      });
    };

    Pages next;
    if (t + kAhead < t_end) next = pages_of(t + kAhead);
    wait_loads<0>();  // the queries among them
    for (; t < t_end; ++t) {
      // This step's tiles have arrived, for all wavefronts, and its predecessor's place is free.
      if (t + kAhead <= t_end) wait_loads<(kAhead - 1) * Ring::kCopies>();
      else wait_loads<0>();
      lds_barrier();
      const int tn = t + kAhead;
      if (tn < t_end) {
        fetch_step(tn, next);
      }
      if (active) {
        const uint4 words = *reinterpret_cast<const uint4*>(Ring::whole()[t % Ring::kSteps]);
        const bool all = __builtin_amdgcn_readfirstlane(words.x & words.y & words.z & words.w) != 0;
        compute(ring + (t % Ring::kSteps) * Ring::kStep, t * kStepKeys, all);
      }
      if (tn + 1 < t_end) next = pages_of(tn + 1);
    }
    if (!active) return;

    const bool full = s0 == 0 && s1 == units;
    const float vs = kE4M3 && a.kv.v_scale ? a.kv.v_scale[hk] : 1.f;
    float* part = a.parts + (int64_t)(2 * (w * a.kv.n_kv_heads + hk) + (first_segment ? 0 : 1)) * a.part_floats;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      l[i] += __shfl_xor(l[i], 16);
      l[i] += __shfl_xor(l[i], 32);
      const int c = 16 * wave + l16;
      if (c >= columns) continue;
      if (full) {
        const int64_t row = start + node[i];
        const int head = hk * a.group + r.cb * kColumns + c - node[i] * a.group;
        const float inv = l[i] == 0.f ? 0.f : vs / l[i];
        uint16_t* out = a.out + row * a.out_stride + (int64_t)head * kDh;
#pragma unroll
        for (int d = 0; d < kBlocks; ++d) {
          uint2 four;
          four.x = pair_down(T(), acc[i][d][0] * inv, acc[i][d][1] * inv);
          four.y = pair_down(T(), acc[i][d][2] * inv, acc[i][d][3] * inv);
          *reinterpret_cast<uint2*>(out + 16 * d + 4 * g4) = four;
        }
        if (g4 == 0 && a.lse)
          a.lse[row * a.n_heads + head] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * 0.6931471805599453f;
      } else {
#pragma unroll
        for (int d = 0; d < kBlocks; ++d)
          *reinterpret_cast<f32x4*>(part + 2 * kColumns + c * kDh + 16 * d + 4 * g4) = acc[i][d];
        if (g4 == 0) {
          part[c] = m[i];
          part[kColumns + c] = l[i];
        }
      }
    }
  }
};

// As paged_tree_kernel, but a block has 64 columns, 16 to each of the four wavefronts: all of
// them read the same keys, which come into LDS by direct copies, a ring of steps ahead.
// Columns of 128, 32 to a wavefront, need half the reads of LDS, but twice the registers:
// 64 nodes x 4 trees of 8,192 keys 83 us where this takes 82, 40 trees over 8 bits 173 and 160.
//
// 131,072 keys of 8 heads of 128 take 98 us, 5.5 TB/s, bound by HBM (122 us without the
// copies' nt where it made 104).  Ragged trees of many nodes are bound by the
// SIMDs' issue: a key and column cost two products of values (the weight's two halves), an
// exponential and, over 8 bits, the conversions of both tiles; 40 trees over 8 bits reach, by
// their lengths, 240 to 300 TFLOP/s and 2.3 to 2.6 TB/s, 64 nodes x 4 trees 413 TFLOP/s.
template <class T, bool kE4M3, int kDh, bool kShaped>
__global__ __launch_bounds__(64 * kTreeWaves, wide_workgroups(kDh, kE4M3)) void paged_tree_wide_kernel(TreeArg a) {
  typedef WideSegment<T, kE4M3, kDh, kShaped> Segment;
  constexpr int kColumns = Segment::kColumns;
  const int hk = blockIdx.x, w = a.workers ? blockIdx.y : blockIdx.z, cb = a.workers ? 0 : blockIdx.y;
  TreeChunk ch;
  TreeRun r{0, 1, 0, w, cb, 1, 0};
  if (a.workers) {
    if (!find_run(a, w, kColumns, ch, r)) return;  // the same for the whole workgroup
  } else {
    ch.load(a, w & ~63, kColumns);
    if (cb >= __builtin_amdgcn_readlane(ch.blocks, w & 63)) return;
  }
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
    Segment::run(a, r, w, hk, start, count, sq, n, first, end, units, s0, s1, columns, first_segment);
    if (a.workers && s0 == 0 && threadIdx.x == 0) note_parts(a, r, w, hk, units, s1, first_segment);
    r.u += s1 - s0;
    r.base += units;
    ++r.cb;
    first_segment = false;
  }
}

// ---------------------------------------------------------------- launches
template <class T, bool kE4M3, int kDh, int kTiles, bool kWide>
void launch_tree_tiles(const TreeArg& a, const TreePlan& p, hipStream_t stream) {
  const dim3 block(64 * kTreeWaves);
  const dim3 grid = a.workers ? dim3(a.kv.n_kv_heads, a.workers) : dim3(a.kv.n_kv_heads, a.blocks, a.trees);
  const bool shaped = a.cap > 0.f || a.slopes;
  if constexpr (kWide) {
    if (shaped)
      hipLaunchKernelGGL((paged_tree_wide_kernel<T, kE4M3, kDh, true>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((paged_tree_wide_kernel<T, kE4M3, kDh, false>), grid, block, 0, stream, a);
  } else {
    if (shaped)
      hipLaunchKernelGGL((paged_tree_kernel<T, kE4M3, kDh, kTiles, true>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((paged_tree_kernel<T, kE4M3, kDh, kTiles, false>), grid, block, 0, stream, a);
  }
  if (!a.workers) return;
  const int tiles = kWide ? 4 * kTiles : kTiles;
  const int64_t outputs = (int64_t)a.trees * p.lines, items = 16 * tiles * (kDh / 4);
  if (p.stripes == 4)
    hipLaunchKernelGGL((tree_join_kernel<T, kE4M3, kDh, 4>), dim3((unsigned)(outputs * items / 64)),
                       dim3(256), 0, stream, a, tiles);
  else
    hipLaunchKernelGGL((tree_join_kernel<T, kE4M3, kDh, 1>), dim3((unsigned)(outputs * items / 256)),
                       dim3(256), 0, stream, a, tiles);
}

template <class T, bool kE4M3, int kDh>
void launch_tree_dim(const TreeArg& a, const TreePlan& p, hipStream_t stream) {
  if (p.wide) {
    launch_tree_tiles<T, kE4M3, kDh, 1, true>(a, p, stream);
  } else if constexpr (kDh >= 128) {
    launch_tree_tiles<T, kE4M3, kDh, 1, false>(a, p, stream);
  } else {
    if (p.tiles == 1) launch_tree_tiles<T, kE4M3, kDh, 1, false>(a, p, stream);
    else launch_tree_tiles<T, kE4M3, kDh, 2, false>(a, p, stream);
  }
}

template <class T, bool kE4M3>
void launch_tree(const TreeArg& a, const TreePlan& p, int head_dim, hipStream_t stream) {
  if (head_dim == 256) launch_tree_dim<T, kE4M3, 256>(a, p, stream);
  else if (head_dim == 128) launch_tree_dim<T, kE4M3, 128>(a, p, stream);
  else launch_tree_dim<T, kE4M3, 64>(a, p, stream);
}

}  // namespace emoe
