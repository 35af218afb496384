// The tree attention's kernel for many columns (exactmoe_drafts.h): wavefronts share
// the keys and take columns of their own.
#pragma once

#include "tree.h"

namespace emoe {

// Wait until this wavefront's loads have arrived, in registers and in LDS.
__device__ __forceinline__ void wait_all_loads() {
  __builtin_amdgcn_s_waitcnt((0x7 << 4) | (0xF << 8));  // vmcnt(0) only
}
// Workgroup barrier that orders LDS accesses but does not wait for loads.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xF | (0x3 << 14) | (0x7 << 4));  // lgkmcnt(0) only
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Keys and values of one step of a workgroup.  Row r of a key holds its 16-byte
// chunks in the order c ^ swizzle(r), so that lanes that read the same chunk of
// neighbouring keys use all banks.
template <int kDh, bool kE4M3>
struct WideStage {
  static constexpr int kRow = kDh * (kE4M3 ? 1 : 2);
  static constexpr int kKeys = kRow == 512 ? 32 : 64;
  uint8_t k[kKeys * kRow], v[kKeys * kRow];

  __device__ static __forceinline__ int swizzle(int row) { return kRow == 64 ? (row >> 1) & 3 : row & 7; }
};
// Stage S of two, one LDS variable each: the compiler waits for copies into a
// variable before reads of that variable only.
template <class Stage, int S>
__device__ __forceinline__ Stage& wide_stage() {
  __shared__ __attribute__((aligned(1024))) Stage stage;
  return stage;
}

template <int kDh, bool kE4M3>
constexpr int wide_keys() { return WideStage<kDh, kE4M3>::kKeys; }

// One block of columns of a tree over a run of its keys, of which this wavefront has
// the tiles wave, wave + 4 .. of 16 columns.
template <class T, bool kE4M3, int kDh, int kTiles, bool kShaped>
struct WideSegment {
  typedef WideTile<T, kE4M3, kDh, kTiles> Tl;
  typedef WideStage<kDh, kE4M3> Stage;
  static constexpr int kRow = Stage::kRow, kKeys = Stage::kKeys, kItem = Tl::kItem;
  static constexpr int kSub = kE4M3 ? 2 : 1;         // steps of a 16-byte chunk of keys
  static constexpr int kChunks = kRow / 64;          // chunks of a lane
  static constexpr int kLaneBytes = Tl::kVWords * 4 > 16 ? 16 : Tl::kVWords * 4;  // of values, at once

  // Dimension of the first element that lane group g has of step s.
  __device__ static __forceinline__ int q_dim(int s, int g) {
    return (16 / kItem) * (4 * (s / kSub) + g) + 8 * (s % kSub);
  }

  // Copies the wavefront's quarter of a stage's rows; `page` is the page of the
  // stage's octet that the lane stands for.
  template <class St>
  __device__ static __forceinline__ void fetch(const TreeArg& a, St& stage, const uint8_t* kbase,
                                               const uint8_t* vbase, int key0, int page, int wave, int lane) {
    constexpr int kRows = kKeys / 4, kRowsAtOnce = 1024 / kRow, kLoads = kRows / kRowsAtOnce;
    const int slot_mask = (1 << a.kv.page_log2) - 1;
    const int in = lane / (kRow / 16), chunk = lane % (kRow / 16);
    auto octet_at = [&](int row) -> int64_t {
      const int p = __builtin_amdgcn_readlane(page, row >> 3);
      return ((uint32_t)p < (uint32_t)a.kv.n_pages ? p : 0) * a.kv.page_bytes +
             (int64_t)((key0 + row) & slot_mask) * a.kv.slot_bytes;
    };
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = __builtin_amdgcn_readfirstlane(kRows * wave + i * kRowsAtOnce);
      int64_t at = octet_at(row);
      if constexpr (kRowsAtOnce == 16) {
        const int64_t second = octet_at(row + 8);
        at = lane >= 32 ? second : at;
      }
      const uint32_t off = (in & 7) * a.kv.slot_bytes +
                           16 * (chunk ^ Stage::swizzle((i * kRowsAtOnce & 7) + in));
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(kbase + at + off),
          (__attribute__((address_space(3))) void*)&stage.k[row * kRow], 16, 0, 0);
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(vbase + at + off),
          (__attribute__((address_space(3))) void*)&stage.v[row * kRow], 16, 0, 0);
    }
  }

  __device__ static __forceinline__ void run(const TreeArg& a, const TreeRun& r, int w, int hk, int start,
                                             int count, int sq, int n, int first, int end, int units, int s0,
                                             int s1, int columns, int block_columns, bool first_segment) {
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g4 = lane >> 4;
    // What each node sees, and its depth: node i's in lane i.
    uint64_t sees = 0;
    if (lane < count) sees = a.tree ? a.tree[start + lane] : (2ull << lane) - 1;
    const int depth = __popcll(sees & ((1ull << lane) - 1));
    const int deepest = a.window > 0 ? (int)wave_reduce_u32<true>((uint32_t)(lane < count ? depth : 0)) : 0;
    const bool active = 16 * wave < columns;

    float scale = a.scale;
    if (!kShaped) scale *= 1.4426950408889634f;
    if (kE4M3 && a.kv.k_scale) scale *= a.kv.k_scale[hk];
    const uint32_t flip = scale < 0.f ? 0x80008000u : 0u;
    scale = fabsf(scale);
    int node[kTiles], deep_at[kTiles];
    float slope[kTiles];
    uint4 q[kTiles][Tl::kSteps];
    f32x4 acc[kTiles][Tl::kDims];
    float m[kTiles], l[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int c = 16 * (wave + 4 * i) + l16, col = r.cb * block_columns + c;
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
      for (int c = 0; c < Tl::kDims; ++c) acc[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float inv_cap = kShaped && a.cap > 0.f ? 1.f / a.cap : 0.f;
    const uint8_t* kbase = a.kv.k + (int64_t)hk * a.kv.head_bytes;
    const uint8_t* vbase = a.kv.v + (int64_t)hk * a.kv.head_bytes;
    const int32_t* table = a.table + (int64_t)sq * a.table_stride;
    const int low = a.window > 0 ? max(0, n + deepest + 1 - a.window) : 0, high = min(n, end);

    // A lane's places in a stage: its keys' chunks (even and odd), its values' part of
    // the rows 4 g4 + 0 .. 3.
    int k_at[2], v_at[4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      k_at[i] = l16 * kRow + 16 * ((g4 | (kRow == 64 ? 0 : 4 * i)) ^ Stage::swizzle(l16));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * g4 + i, byte = kLaneBytes * l16;
      v_at[i] = row * kRow + 16 * ((byte >> 4) ^ Stage::swizzle(row)) + (byte & 15);
    }

    auto compute = [&](const Stage& stage, int t, uint32_t there_octets) __attribute__((always_inline)) {
#pragma unroll
      for (int sub = 0; sub < kKeys / 32; ++sub) {
        const int key0 = t * kKeys + 32 * sub;
        if (key0 >= end || key0 + 32 <= first) continue;
        f32x4 s[kTiles][2];
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) s[i][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < kChunks; ++p)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 c = *reinterpret_cast<const uint4*>(stage.k + k_at[p & 1] + (32 * sub + 16 * h) * kRow +
                                                            128 * (p >> 1));
            if constexpr (kE4M3) {
              typedef typename Tl::H16 H;
              const uint4 x0 = make_uint4(H::template from_e4m3<false>(c.x), H::template from_e4m3<true>(c.x),
                                          H::template from_e4m3<false>(c.y), H::template from_e4m3<true>(c.y));
              const uint4 x1 = make_uint4(H::template from_e4m3<false>(c.z), H::template from_e4m3<true>(c.z),
                                          H::template from_e4m3<false>(c.w), H::template from_e4m3<true>(c.w));
#pragma unroll
              for (int i = 0; i < kTiles; ++i) {
                s[i][h] = H::mfma(x0, q[i][2 * p], s[i][h]);
                s[i][h] = H::mfma(x1, q[i][2 * p + 1], s[i][h]);
              }
            } else {
#pragma unroll
              for (int i = 0; i < kTiles; ++i) s[i][h] = Tl::H16::mfma(c, q[i][p], s[i][h]);
            }
          }
        Tl tile;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint8_t* at = stage.v + v_at[j & 3] + (32 * sub + 16 * (j >> 2)) * kRow;
          if constexpr (Tl::kVWords == 1) {
            tile.v[j][0] = *reinterpret_cast<const uint32_t*>(at);
          } else if constexpr (Tl::kVWords == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(at);
            tile.v[j][0] = x.x, tile.v[j][1] = x.y;
          } else {
#pragma unroll
            for (int u = 0; u < Tl::kVWords / 4; ++u) {
              const uint4 x = *reinterpret_cast<const uint4*>(at + 256 * u);
              tile.v[j][4 * u] = x.x, tile.v[j][4 * u + 1] = x.y, tile.v[j][4 * u + 2] = x.z,
                         tile.v[j][4 * u + 3] = x.w;
            }
          }
        }
        auto key_of = [&](int j, int group) { return key0 + 16 * (j >> 2) + 4 * group + (j & 3); };
        float z[kTiles][8], p[kTiles][8];
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) z[i][j] = kShaped ? s[i][j >> 2][j & 3] * scale : s[i][j >> 2][j & 3];
        if constexpr (kShaped) {
          int key_at[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) key_at[j] = key_of(j, g4) - n;
          shape_scores(z, a.cap, inv_cap, a.slopes != nullptr, slope, deep_at, key_at, key0 + 32 > n, depth);
        }
        const uint32_t octets = (there_octets >> (4 * sub)) & 15;
        uint32_t bad = 0;
        const bool masked = !(key0 >= low && key0 + 32 <= high && octets == 15);
        if (masked) {
          uint32_t there = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int key = key_of(j, g4);
            if (key >= first && key < end && (octets >> (2 * (j >> 2) + (g4 >> 1))) & 1) there |= 1u << j;
          }
          bad = tile.not_finite() & there;
          bad |= __shfl_xor(bad, 1);
          bad |= __shfl_xor(bad, 2);
          bad |= __shfl_xor(bad, 4);
          bad |= __shfl_xor(bad, 8);
          tile.clear_v(there & ~bad);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int key_at = key_of(j, g4) - n, key_depth = __shfl(depth, key_at & 63);
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
              const uint64_t mask = __shfl(sees, node[i]);
              const int deep = __shfl(depth, node[i]);
              if (!((there >> j) & 1) || !node_sees(mask, deep, key_at, key_depth, a.window)) z[i][j] = -INFINITY;
            }
          }
        }
        soft_step<Tl>(z, kShaped ? 1.f : scale, masked, m, l, acc, p);
        if (__any(bad != 0)) {
          for (int x = 0; x < 32; ++x) {
            const int j = x & 7, kg = x >> 3, key = key_of(j, kg);
            if (!((__builtin_amdgcn_readlane((int)bad, 16 * kg) >> j) & 1)) continue;
            const uint8_t* row = vbase + table[key >> a.kv.page_log2] * a.kv.page_bytes +
                                 (int64_t)(key & ((1 << a.kv.page_log2) - 1)) * a.kv.slot_bytes;
            const int key_depth = __shfl(depth, (key - n) & 63);
            bool seen[kTiles];
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
              seen[i] = node_sees(__shfl(sees, node[i]), __shfl(depth, node[i]), key - n, key_depth, a.window);
            add_one_key<T, kE4M3, Tl>(row, j, kg, p, seen, acc);
          }
        }
        add_weighted(tile, p, acc);
      }
    };

    const int t_all = (end + kKeys - 1) / kKeys, t0 = first / kKeys;
    int t = t0 + s0;
    const int t_end = a.workers ? min(t0 + s1, t_all) : t_all;
    auto page_of = [&](int tile) -> int {
      const int key = tile * kKeys + 8 * lane;
      return lane < kKeys / 8 && tile < t_end && key < end ? table[key >> a.kv.page_log2] : -1;
    };
    auto octets_of = [&](int page) -> uint32_t {
      return (uint32_t)__ballot((uint32_t)page < (uint32_t)a.kv.n_pages) & ((1u << (kKeys / 8)) - 1);
    };
    lds_barrier();  // the last segment's readers are done
    if (t < t_end) {
      Stage &st0 = wide_stage<Stage, 0>(), &st1 = wide_stage<Stage, 1>();
      int page = page_of(t);
      uint32_t now = octets_of(page);
      fetch(a, st0, kbase, vbase, t * kKeys, page, wave, lane);
      page = page_of(t + 1);
      // The copies of the next step are under way while this one is computed.
      auto step = [&](const Stage& here, Stage& there) __attribute__((always_inline)) -> bool {
        wait_all_loads();
        lds_barrier();
        const uint32_t next = octets_of(page);
        if (t + 1 < t_end) fetch(a, there, kbase, vbase, (t + 1) * kKeys, page, wave, lane);
        page = page_of(t + 2);
        if (active) compute(here, t, now);
        now = next;
        return ++t < t_end;
      };
      while (step(st0, st1) && step(st1, st0)) {
      }
    }
    if (!active) return;

    const bool full = s0 == 0 && s1 == units;
    const float vs = kE4M3 && a.kv.v_scale ? a.kv.v_scale[hk] : 1.f;
    float* part = a.parts + (int64_t)(2 * (w * a.kv.n_kv_heads + hk) + (first_segment ? 0 : 1)) * a.part_floats;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      l[i] += __shfl_xor(l[i], 16);
      l[i] += __shfl_xor(l[i], 32);
      const int c = 16 * (wave + 4 * i) + l16;
      if (c >= columns) continue;
      if (full) {
        const int64_t row = start + node[i];
        const int head = hk * a.group + r.cb * block_columns + c - node[i] * a.group;
        const float inv = l[i] == 0.f ? 0.f : vs / l[i];
        uint16_t* out = a.out + row * a.out_stride + (int64_t)head * kDh;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int d = 0; d < Tl::kDims; d += 4) {
            uint2 four;
            four.x = T::down(acc[i][d][x] * inv) | (T::down(acc[i][d + 1][x] * inv) << 16);
            four.y = T::down(acc[i][d + 2][x] * inv) | (T::down(acc[i][d + 3][x] * inv) << 16);
            *reinterpret_cast<uint2*>(out + Tl::out_dim(4 * g4 + x, d)) = four;
          }
        if (g4 == 0 && a.lse)
          a.lse[row * a.n_heads + head] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * 0.6931471805599453f;
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int d = 0; d < Tl::kDims; d += 4)
            *reinterpret_cast<float4*>(part + 2 * block_columns + c * kDh + Tl::out_dim(4 * g4 + x, d)) =
                make_float4(acc[i][d][x], acc[i][d + 1][x], acc[i][d + 2][x], acc[i][d + 3][x]);
        if (g4 == 0) {
          part[c] = m[i];
          part[block_columns + c] = l[i];
        }
      }
    }
  }
};

// As paged_tree_kernel, but a block has 64 * kTiles columns and its four wavefronts take
// every fourth tile of 16 of them: all of them read the same keys, which come into LDS
// by direct copies, two steps in turn.  A wavefront so has few columns' statistics and
// outputs, and two wavefronts to a SIMD have room for them.
template <class T, bool kE4M3, int kDh, int kTiles, bool kShaped>
__global__ __launch_bounds__(64 * kTreeWaves, 2) void paged_tree_wide_kernel(TreeArg a) {
  constexpr int kColumns = 64 * kTiles;
  int w, hk, cb = 0;
  if (a.workers) {
    w = blockIdx.x / a.kv.n_kv_heads;
    hk = blockIdx.x % a.kv.n_kv_heads;
  } else {
    const int chunk = blockIdx.x / (8 * a.blocks), at = blockIdx.x % (8 * a.blocks);
    const int pairs = min(8, a.trees * a.kv.n_kv_heads - 8 * chunk), pair = 8 * chunk + at % pairs;
    cb = at / pairs;
    w = pair / a.kv.n_kv_heads;
    hk = pair % a.kv.n_kv_heads;
  }
  TreeChunk ch;
  TreeRun r{1, 0, 1, 0, w, cb};
  if (a.workers) {
    if (!find_run(a, w, kColumns, ch, r)) return;  // the same for the whole workgroup
  } else {
    ch.load(a, w & ~63, kColumns);
    if (cb >= __builtin_amdgcn_readlane(ch.blocks, w & 63)) return;
  }
  bool first_segment = true;
  while (r.u < r.u_end) {
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
    if (kTiles > 1 && columns > 64)
      WideSegment<T, kE4M3, kDh, kTiles, kShaped>::run(a, r, w, hk, start, count, sq, n, first, end, units, s0, s1,
                                                       columns, kColumns, first_segment);
    else
      WideSegment<T, kE4M3, kDh, 1, kShaped>::run(a, r, w, hk, start, count, sq, n, first, end, units, s0, s1,
                                                  columns, kColumns, first_segment);
    if (a.workers && s0 == 0 && threadIdx.x == 0) {
      int32_t* h = a.heads_of + 3 * (((int64_t)r.tr * a.blocks + r.cb) * a.kv.n_kv_heads + hk);
      h[0] = w;
      h[1] = s1 == units ? 0 : (r.base + units - 1) / r.run - w + 1;
      h[2] = first_segment ? 0 : 1;
    }
    r.u += s1 - s0;
    r.base += units;
    ++r.cb;
    first_segment = false;
  }
}

// ---------------------------------------------------------------- launches
template <class T, bool kE4M3, int kDh, int kTiles, bool kWide>
void launch_tree_tiles(const TreeArg& a, const TreePlan& p, hipStream_t stream) {
  const int64_t grid_x = a.workers ? (int64_t)a.workers * a.kv.n_kv_heads : (int64_t)a.trees * p.lines;
  const dim3 grid((unsigned)grid_x), block(64 * kTreeWaves);
  const bool shaped = a.cap > 0.f || a.slopes;
  if constexpr (kWide) {
    if (shaped)
      hipLaunchKernelGGL((paged_tree_wide_kernel<T, kE4M3, kDh, kTiles, true>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((paged_tree_wide_kernel<T, kE4M3, kDh, kTiles, false>), grid, block, 0, stream, a);
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
    if constexpr (kDh == 256) {
      launch_tree_tiles<T, kE4M3, kDh, 1, true>(a, p, stream);
    } else {
      if (p.tiles == 4) launch_tree_tiles<T, kE4M3, kDh, 1, true>(a, p, stream);
      else launch_tree_tiles<T, kE4M3, kDh, 2, true>(a, p, stream);
    }
  } else if constexpr (kDh == 256) {
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
