// Acceptance of drafted tokens, and the moves of keys and values that follow:
// compaction and forks of sequences in all layers' caches (exactmoe_drafts.h).
#include "exactmoe_drafts.h"
#include "paged.h"

using namespace emoe;

namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- acceptance
struct AcceptArg {
  const int32_t *tokens, *chosen, *starts, *lengths;
  const uint64_t* tree;
  int32_t *path, *accepted, *new_tokens, *new_lengths;
  int64_t path_stride, new_tokens_stride;
  int32_t rows, trees, max_nodes;
};

// A wavefront takes a tree, a lane a node; a step of the walk is a ballot.  Bound
// by the chain of two trips to memory and, per accepted node, about 30 cycles: one tree of
// 26 nodes takes 2.1 us, 500 trees of up to 64 nodes 3.3.
__global__ __launch_bounds__(kThreads) void accept_kernel(AcceptArg a) {
  const int lane = lane_id(), g = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (g >= a.trees) return;
  int start = g * a.max_nodes;
  int64_t count = a.max_nodes;
  if (a.starts) {
    start = a.starts[g];
    count = (int64_t)a.starts[g + 1] - start;
    if (start < 0 || start > a.rows) start = a.rows;
  }
  const int nodes = (int)max((int64_t)0, min(count, (int64_t)min(a.max_nodes, a.rows - start)));
  int token = -1, chosen = -1, parent = -1;
  if (lane < nodes) {
    token = a.tokens[start + lane];
    chosen = a.chosen[start + lane];
    const uint64_t sees = a.tree ? a.tree[start + lane] : ~0ull;
    parent = 63 - __builtin_clzll((sees & ((1ull << lane) - 1)) << 1 | 1) - 1;
  }
  int path = -1, made = -1, m = 0;
  for (int at = 0; m < nodes; ++m) {
    const int want = __builtin_amdgcn_readlane(chosen, at);
    if (lane == m) {
      path = at;
      made = want;
    }
    const uint64_t next = __ballot(lane < nodes && parent == at && token == want && want >= 0);
    if (next == 0) {
      ++m;
      break;
    }
    at = __builtin_ctzll(next);
  }
  if (lane < a.max_nodes) {
    a.path[g * a.path_stride + lane] = path;
    if (a.new_tokens) a.new_tokens[g * a.new_tokens_stride + lane] = made;
  }
  if (lane == 0) {
    a.accepted[g] = m;
    if (a.new_lengths) a.new_lengths[g] = a.lengths[g] + m;
  }
}

// ---------------------------------------------------------------- moves
constexpr int kLayers = 64;  // caches of one launch

// Where the layers' keys and values are; strides in bytes, and what of a slot is
// its own: pieces of 16 bytes of each head.
struct LayersArg {
  uint8_t* pages[2 * kLayers];  // k, v, k, v ..
  int64_t page_bytes;
  int32_t slot_bytes, head_bytes, n_pages, page_log2, n_kv_heads, piece_log2, layers;
  bool slots_inside;
};

struct CompactArg {
  LayersArg kv;
  const int32_t *lengths, *path, *accepted, *seqs, *table;
  int64_t path_stride, table_stride;
  int32_t max_nodes, n_seqs, table_width, blocks;
};

__device__ __forceinline__ int64_t slot_offset(const LayersArg& kv, const int32_t* table, int64_t position,
                                               int table_width) {
  const int64_t col = position >> kv.page_log2;
  if (col >= table_width) return -1;
  const int page = table[col];
  if ((uint32_t)page >= (uint32_t)kv.n_pages) return -1;
  return page * kv.page_bytes + (position & ((1 << kv.page_log2) - 1)) * kv.slot_bytes;
}

// A thread takes one piece of 16 bytes of a head, of keys or values of a layer, and
// makes all of the tree's moves of it in turn, eight at a time: their loads, then their
// stores.  The source of a move lies behind the targets of the moves before it (path[i] > i),
// so what is read has not been written by this call.
// The compiler keeps the eight pieces in scratch memory (144 bytes a thread) and waits for
// each load before the next: 61 trees of 24 MB in 28 layers take 9.9 us, 2.5 TB/s.  Small calls
// are bound by the chain lengths, path, page table, keys: 4.1 us for one tree in 16 layers.
__global__ __launch_bounds__(kThreads) void compact_kernel(CompactArg a) {
  __shared__ int64_t from[64], to[64];
  __shared__ int moves;
  const int g = blockIdx.x / a.blocks, tid = threadIdx.x;
  const int item = (blockIdx.x % a.blocks) * kThreads + tid, per = a.kv.n_kv_heads << a.kv.piece_log2;
  const int which = item / per, rest = item % per;
  const int64_t in_slot =
      (int64_t)(rest >> a.kv.piece_log2) * a.kv.head_bytes + 16 * (rest & ((1 << a.kv.piece_log2) - 1));
  uint8_t* base = a.kv.pages[min(which, 2 * a.kv.layers - 1)] + in_slot;  // on its way with the moves
  if (tid < 64) {
    const int s = a.seqs ? a.seqs[g] : g, n = a.lengths[g];
    const int count = min(a.accepted[g], a.max_nodes);
    int64_t src = -1, dst = -1;
    if ((uint32_t)s < (uint32_t)a.n_seqs && n >= 0 && tid < count) {
      const int p = a.path[g * a.path_stride + tid];
      if (p > tid) {
        const int32_t* table = a.table + (int64_t)s * a.table_stride;
        src = slot_offset(a.kv, table, (int64_t)n + p, a.table_width);
        dst = slot_offset(a.kv, table, (int64_t)n + tid, a.table_width);
      }
    }
    const bool yes = src >= 0 && dst >= 0;
    const uint64_t all = __ballot(yes);
    const int at = __popcll(all & ((1ull << tid) - 1));
    if (yes) {
      from[at] = src;
      to[at] = dst;
    }
    if (tid == 0) moves = __popcll(all);
  }
  __syncthreads();
  if (which >= 2 * a.kv.layers) return;
  for (int i0 = 0; i0 < moves; i0 += 8) {
    uint4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i0 + i < moves) x[i] = *reinterpret_cast<const uint4*>(base + from[i0 + i]);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i0 + i < moves) *reinterpret_cast<uint4*>(base + to[i0 + i]) = x[i];
  }
}

struct ForkArg {
  LayersArg kv;
  const int32_t *table, *parents, *lengths, *fresh;
  int32_t* new_table;
  int64_t table_stride, new_table_stride;
  int32_t forks, n_seqs, table_width, table_blocks, copy_blocks;
};

constexpr int kForkPieces = 4;  // of a thread

// Workgroups of the new tables (table_blocks to a fork), then those of the copies:
// copy_blocks to a fork, layer and side, each of up to 1,024 pieces of 16 bytes in
// the order in which they lie in memory.  Bound by HBM, each byte read and written
// once: 200 forks, 60 MB read and written, take 25 us, 4.7 TB/s, 93% of a large copy's
// rate; small calls by the chain parent, page table, keys: 4 forks 5.4 us.
__global__ __launch_bounds__(kThreads) void fork_kernel(ForkArg a) {
  const int tid = threadIdx.x, ps = 1 << a.kv.page_log2;
  int64_t b = blockIdx.x;
  const bool tables = b < (int64_t)a.forks * a.table_blocks;
  if (!tables) b -= (int64_t)a.forks * a.table_blocks;
  const int per_fork = tables ? a.table_blocks : a.copy_blocks * 2 * a.kv.layers;
  const int f = (int)(b / per_fork), sub = (int)(b % per_fork);
  const int parent = a.parents[f];
  int n = a.lengths[f];
  const int fresh = a.fresh ? a.fresh[f] : -1;
  const bool valid = (uint32_t)parent < (uint32_t)a.n_seqs && n > 0;
  n = valid ? (int)min((int64_t)n, (int64_t)a.table_width << a.kv.page_log2) : 0;
  const int last = n >> a.kv.page_log2, part = n & (ps - 1);
  const int32_t* row = a.table + (int64_t)(valid ? parent : 0) * a.table_stride;
  const bool copies = part > 0 && (uint32_t)fresh < (uint32_t)a.kv.n_pages;
  if (tables) {
    for (int64_t c = sub * kThreads + tid; c < a.table_width; c += a.table_blocks * kThreads) {
      int page = -1;
      if (c < last || (c == last && part > 0)) {
        page = row[c];
        if (c == last && copies && (uint32_t)page < (uint32_t)a.kv.n_pages) page = fresh;
      }
      a.new_table[(int64_t)f * a.new_table_stride + c] = page;
    }
    return;
  }
  if (!copies) return;
  const int page = row[last];
  if ((uint32_t)page >= (uint32_t)a.kv.n_pages || page == fresh) return;
  uint8_t* base = a.kv.pages[sub / a.copy_blocks];
  const uint8_t* src = base + page * a.kv.page_bytes;
  uint8_t* dst = base + fresh * a.kv.page_bytes;
  const int first = (sub % a.copy_blocks) * kForkPieces * kThreads + tid;
  const int items = part * a.kv.n_kv_heads << a.kv.piece_log2, pieces = (1 << a.kv.piece_log2) - 1;
  uint4 x[kForkPieces];
  int64_t at[kForkPieces];
#pragma unroll
  for (int i = 0; i < kForkPieces; ++i) {
    const int item = first + i * kThreads;
    if (item >= items) continue;
    const int line = item >> a.kv.piece_log2;
    const int slot = a.kv.slots_inside ? line % part : line / a.kv.n_kv_heads;
    const int head = a.kv.slots_inside ? line / part : line % a.kv.n_kv_heads;
    at[i] = (int64_t)slot * a.kv.slot_bytes + (int64_t)head * a.kv.head_bytes + 16 * (item & pieces);
    x[i] = load_once(reinterpret_cast<const uint4*>(src + at[i]));
  }
#pragma unroll
  for (int i = 0; i < kForkPieces; ++i)
    if (first + i * kThreads < items) *reinterpret_cast<uint4*>(dst + at[i]) = x[i];
}

// ---------------------------------------------------------------- the host's side
int32_t check_layers(const emoe_paged_kv* kv, int32_t n_layers) {
  if (n_layers < 1) return report_error(EMOE_EINVAL, "n_layers %d", n_layers);
  int32_t st = check_kv(kv);
  if (st) return st;
  for (int i = 1; i < n_layers; ++i) {
    if ((st = check_kv(kv + i))) return st;
    const emoe_paged_kv &a = kv[0], &b = kv[i];
    if (a.dtype != b.dtype || a.n_pages != b.n_pages || a.page_size != b.page_size ||
        a.n_kv_heads != b.n_kv_heads || a.head_dim != b.head_dim || a.page_stride != b.page_stride ||
        a.slot_stride != b.slot_stride || a.head_stride != b.head_stride)
      return report_error(EMOE_ESHAPE, "cache %d has another type, size or stride than the first one", i);
  }
  // The same place twice would be moved twice, at once.
  auto place = [&](int64_t i) { return i & 1 ? kv[i >> 1].v_pages : kv[i >> 1].k_pages; };
  for (int64_t i = 1; i < 2 * (int64_t)n_layers; ++i)
    for (int64_t j = 0; j < i; ++j)
      if (place(i) == place(j))
        return report_error(EMOE_EINVAL, "caches %d and %d have pages at the same place", (int)(j >> 1), (int)(i >> 1));
  return EMOE_OK;
}

// Those of layers l0 .. on, as many as a launch takes.
LayersArg layers_of(const emoe_paged_kv* kv, int32_t n_layers, int32_t l0) {
  const KvView v = view_of(kv[0]);
  LayersArg a;
  a.layers = n_layers - l0 < kLayers ? n_layers - l0 : kLayers;
  for (int i = 0; i < a.layers; ++i) {
    a.pages[2 * i] = static_cast<uint8_t*>(kv[l0 + i].k_pages);
    a.pages[2 * i + 1] = static_cast<uint8_t*>(kv[l0 + i].v_pages);
  }
  a.page_bytes = v.page_bytes;
  a.slot_bytes = v.slot_bytes;
  a.head_bytes = v.head_bytes;
  a.n_pages = v.n_pages;
  a.page_log2 = v.page_log2;
  a.n_kv_heads = v.n_kv_heads;
  const int bytes = kv[0].head_dim * (kv[0].dtype == EMOE_E4M3 ? 1 : 2);
  a.piece_log2 = __builtin_ctz((unsigned)bytes / 16);
  a.slots_inside = v.head_bytes > v.slot_bytes;
  return a;
}

int32_t check_table(const int32_t* table, int32_t n_seqs, int32_t table_width, int64_t table_stride) {
  if (n_seqs < 0 || table_width < 0) return report_error(EMOE_EINVAL, "negative n_seqs or table_width");
  if (n_seqs > 0 && table_width > 0 && !table) return report_error(EMOE_EINVAL, "page_table is NULL");
  if (n_seqs > 1 && table_stride < table_width)
    return report_error(EMOE_EINVAL, "table_stride %lld below table_width %d", (long long)table_stride,
                        table_width);
  return EMOE_OK;
}

int32_t check_nodes(int32_t max_nodes) {
  if (max_nodes < 1 || max_nodes > EMOE_MAX_NODES)
    return report_error(EMOE_ESHAPE, "max_nodes %d: need 1 to %d", max_nodes, EMOE_MAX_NODES);
  return EMOE_OK;
}

constexpr int64_t kMostBlocks = ((int64_t)1 << 32) / kThreads - 1;  // a grid has fewer than 2^32 threads

}  // namespace

extern "C" {

int32_t emoe_accept_drafts(const emoe_accept_args* args, hipStream_t stream) {
  if (!args) return report_error(EMOE_EINVAL, "args is NULL");
  const emoe_accept_args& A = *args;
  int32_t st = check_nodes(A.max_nodes);
  if (st) return st;
  if (A.rows < 0 || A.trees < 0) return report_error(EMOE_EINVAL, "negative rows or trees (%d, %d)", A.rows, A.trees);
  if (!A.starts && A.rows != (int64_t)A.trees * A.max_nodes)
    return report_error(EMOE_ESHAPE, "%d rows without starts: need %d trees of %d nodes", A.rows, A.trees,
                        A.max_nodes);
  if (A.trees == 0) return EMOE_OK;
  if (A.rows > 0 && (!A.tokens || !A.chosen)) return report_error(EMOE_EINVAL, "tokens or chosen is NULL");
  if (!A.path || !A.accepted) return report_error(EMOE_EINVAL, "path or accepted is NULL");
  if (A.new_lengths && !A.lengths) return report_error(EMOE_EINVAL, "new_lengths without lengths");
  if (A.trees > 1 && (A.path_stride < A.max_nodes || (A.new_tokens && A.new_tokens_stride < A.max_nodes)))
    return report_error(EMOE_EINVAL, "path_stride %lld or new_tokens_stride %lld below max_nodes %d",
                        (long long)A.path_stride, (long long)A.new_tokens_stride, A.max_nodes);
  AcceptArg a;
  a.tokens = A.tokens;
  a.chosen = A.chosen;
  a.starts = A.starts;
  a.lengths = A.lengths;
  a.tree = A.tree;
  a.path = A.path;
  a.accepted = A.accepted;
  a.new_tokens = A.new_tokens;
  a.new_lengths = A.new_lengths;
  a.path_stride = A.path_stride;
  a.new_tokens_stride = A.new_tokens_stride;
  a.rows = A.rows;
  a.trees = A.trees;
  a.max_nodes = A.max_nodes;
  // Up to 2^24 trees of a wavefront each to a launch (the arrays' strides move along).
  constexpr int32_t kTrees = 1 << 24;
  for (int64_t t0 = 0; t0 < A.trees; t0 += kTrees) {
    if (t0 > 0) {
      if (a.starts) a.starts += kTrees;
      a.path += kTrees * a.path_stride;
      a.accepted += kTrees;
      if (a.new_tokens) a.new_tokens += kTrees * a.new_tokens_stride;
      if (a.lengths) a.lengths += kTrees;
      if (a.new_lengths) a.new_lengths += kTrees;
      if (!a.starts) {
        a.tokens += (int64_t)kTrees * a.max_nodes;
        a.chosen += (int64_t)kTrees * a.max_nodes;
        if (a.tree) a.tree += (int64_t)kTrees * a.max_nodes;
        a.rows -= kTrees * a.max_nodes;
      }
    }
    a.trees = (int32_t)(A.trees - t0 < kTrees ? A.trees - t0 : kTrees);
    hipLaunchKernelGGL(accept_kernel, dim3((unsigned)((a.trees + 3) / 4)), dim3(kThreads), 0, stream, a);
    if ((st = launched("accept_kernel"))) return st;
  }
  return EMOE_OK;
}

int32_t emoe_paged_compact(const emoe_paged_kv* kv, int32_t n_layers, const emoe_compact_args* args,
                           hipStream_t stream) {
  int32_t st = check_layers(kv, n_layers);
  if (st) return st;
  if (!args) return report_error(EMOE_EINVAL, "args is NULL");
  const emoe_compact_args& A = *args;
  if ((st = check_table(A.page_table, A.n_seqs, A.table_width, A.table_stride))) return st;
  if ((st = check_nodes(A.max_nodes))) return st;
  if (A.trees < 0) return report_error(EMOE_EINVAL, "trees %d", A.trees);
  if (A.trees == 0) return EMOE_OK;
  if (!A.lengths || !A.path || !A.accepted)
    return report_error(EMOE_EINVAL, "lengths, path or accepted is NULL");
  if (A.trees > 1 && A.path_stride < A.max_nodes)
    return report_error(EMOE_EINVAL, "path_stride %lld below max_nodes %d", (long long)A.path_stride,
                        A.max_nodes);
  for (int32_t l0 = 0; l0 < n_layers; l0 += kLayers) {
    CompactArg a;
    a.kv = layers_of(kv, n_layers, l0);
    a.table = A.page_table;
    a.table_stride = A.table_stride;
    a.path_stride = A.path_stride;
    a.max_nodes = A.max_nodes;
    a.n_seqs = A.n_seqs;
    a.table_width = A.table_width;
    // A page of 8 slots or more is within 2^30 bytes: at most 2^23 pieces to a slot.
    const int64_t items = (int64_t)2 * a.kv.layers * (a.kv.n_kv_heads << a.kv.piece_log2);
    a.blocks = (int32_t)((items + kThreads - 1) / kThreads);
    const int64_t most = kMostBlocks / a.blocks;
    for (int64_t t0 = 0; t0 < A.trees; t0 += most) {
      const int64_t trees = A.trees - t0 < most ? A.trees - t0 : most;
      if (A.seqs) {
        a.seqs = A.seqs + t0;
      } else {  // tree g of a later launch is of a later sequence
        a.seqs = nullptr;
        a.table = A.page_table + t0 * A.table_stride;
        a.n_seqs = (int32_t)(A.n_seqs - t0 > 0 ? A.n_seqs - t0 : 0);
      }
      a.lengths = A.lengths + t0;
      a.path = A.path + t0 * A.path_stride;
      a.accepted = A.accepted + t0;
      hipLaunchKernelGGL(compact_kernel, dim3((unsigned)(trees * a.blocks)), dim3(kThreads), 0, stream, a);
      if ((st = launched("compact_kernel"))) return st;
    }
  }
  return EMOE_OK;
}

int32_t emoe_paged_fork(const emoe_paged_kv* kv, int32_t n_layers, const emoe_fork_args* args,
                        hipStream_t stream) {
  int32_t st = check_layers(kv, n_layers);
  if (st) return st;
  if (!args) return report_error(EMOE_EINVAL, "args is NULL");
  const emoe_fork_args& A = *args;
  if ((st = check_table(A.page_table, A.n_seqs, A.table_width, A.table_stride))) return st;
  if (A.forks < 0) return report_error(EMOE_EINVAL, "forks %d", A.forks);
  if (A.forks == 0 || A.table_width == 0) return EMOE_OK;
  if (!A.parents || !A.lengths || !A.new_table)
    return report_error(EMOE_EINVAL, "parents, lengths or new_table is NULL");
  if (A.forks > 1 && A.new_table_stride < A.table_width)
    return report_error(EMOE_EINVAL, "new_table_stride %lld below table_width %d",
                        (long long)A.new_table_stride, A.table_width);
  if (A.n_seqs > 0) {
    const int32_t *t = A.page_table, *t_end = t + (A.n_seqs - 1) * (A.n_seqs > 1 ? A.table_stride : 0) + A.table_width;
    const int32_t *c = A.new_table, *c_end = c + (A.forks - 1) * (A.forks > 1 ? A.new_table_stride : 0) + A.table_width;
    if (c < t_end && t < c_end) return report_error(EMOE_EINVAL, "new_table overlaps page_table");
  }
  for (int32_t l0 = 0; l0 < n_layers; l0 += kLayers) {
    ForkArg a;
    a.kv = layers_of(kv, n_layers, l0);
    a.table = A.page_table;
    a.table_stride = A.table_stride;
    a.new_table_stride = A.new_table_stride;
    a.n_seqs = A.n_seqs;
    a.table_width = A.table_width;
    a.table_blocks = l0 > 0 ? 0 : (int32_t)(((int64_t)A.table_width + 8 * kThreads - 1) / (8 * kThreads));
    const int64_t pieces = (int64_t)((kv->page_size - 1) * kv->n_kv_heads) << a.kv.piece_log2;  // below 2^26
    a.copy_blocks = A.fresh ? (int32_t)((pieces + kForkPieces * kThreads - 1) / (kForkPieces * kThreads)) : 0;
    const int64_t per = a.table_blocks + (int64_t)a.copy_blocks * 2 * a.kv.layers;
    if (per == 0) break;
    const int64_t most = kMostBlocks / per;
    for (int64_t f0 = 0; f0 < A.forks; f0 += most) {
      a.forks = (int32_t)(A.forks - f0 < most ? A.forks - f0 : most);
      a.parents = A.parents + f0;
      a.lengths = A.lengths + f0;
      a.fresh = A.fresh ? A.fresh + f0 : nullptr;
      a.new_table = A.new_table + f0 * A.new_table_stride;
      hipLaunchKernelGGL(fork_kernel, dim3((unsigned)(a.forks * per)), dim3(kThreads), 0, stream, a);
      if ((st = launched("fork_kernel"))) return st;
    }
  }
  return EMOE_OK;
}

}  // extern "C"
