// Attention of trees of drafted tokens over a paged cache (exactmoe_drafts.h): the
// call's checks and how its work is cut.  The kernels are in tree.h and tree_wide.h.
#include "tree.h"

using namespace emoe;

namespace {

constexpr int64_t kMostColumns = 1 << 20;  // query heads of a key head, of all nodes: blocks are a grid's second axis
constexpr int kUnits = 256;                // CUs

// Which kernel, and how its work is cut.
//  - Up to 16 columns (32 of 64 dimensions) paged_tree_kernel, whose wavefronts take keys
//    of their own straight from memory to registers; more paged_tree_wide_kernel, whose
//    wavefronts share them.  4 columns, 64 trees of 1,001 keys of 8 heads of 128 49.3 and
//    53.3 us (both cut); 26 columns of 16 heads 17.6 and 13.1 us over 328 keys, 23.9 and 16.6 over 2,026.
//    The bound of a tree's nodes decides, as it does on the number of blocks, since the host knows
//    no other: those 64 rows take 46 us under a bound of 1 and 140 under 64, wide and whole.
//  - An output, that is a block of columns of a tree and key head, has one workgroup where
//    there are few keys; else its keys are cut over the workers of its key head (find_run)
//    and tree_join_kernel joins the parts in a launch of its own.
//    Whole and cut: 328 keys of 16 heads 18.3 and 12.8 us, 226 keys 13.4 and 12.6, but 20 trees
//    of 216 keys 11.0 and 17.0 (wide); 504 keys, 16 columns 11.5 and 12.2 (not wide); 640
//    outputs of up to 16,384 563 and 160.  Few are twice as many keys where every CU has an
//    output, 320 of 316 keys 22.4 and 26.2 us, 960 of up to 506 44 and 63 (wide), 480 of up to
//    1,004 28 and 33 (not wide); but not of shaped scores, whose steps are longer: 280 of up to
//    496 39 and 31, of 492 41 and 38.
//  - From 1,024 outputs on few are up to 2,048 keys: whole outputs fill the CUs several times,
//    and what is left is that the longest one may come last.  128 ragged trees, 8 key heads of
//    128, whole and cut: 16 nodes each (wide) over up to 600 keys 49 and 64 us, 1,000 67 and 78,
//    2,000 106 and 110, 3,000 144 and 133, 4,096 187 and 166, 16,384 646 and 467; one node (not
//    wide) 1,000 42 and 46, 2,000 72 and 68, 3,000 101 and 94, 16,384 523 and 387; one of 131,072
//    keys among short ones 3,590 and 192, of one node 1,448 and 138.  400 trees of 2,000 keys 260
//    and 290, 4,096 468 and 472, 16,384 1,619 and 1,473.  Trees of equal lengths lose about 1%
//    (128 of 8,000 keys 702 and 706 us) or win what the last turn of whole ones leaves idle (130 of
//    8,000 883 and 755).  Against the rule are shaped scores of up to 2,000 keys (300 trees of 4
//    key heads of 64 269 and 163), and thousands of trees of one key head, whose lengths every
//    worker looks through (3,000 of up to 6,000 keys 487 and 548).  With key heads so many that
//    fewer than 8 workers belong to each, outputs fill the CUs more evenly than workers.
TreePlan tree_plan(const emoe_paged_kv& kv, int32_t trees, int32_t n_heads, int64_t max_keys,
                   int32_t max_nodes, int32_t window, bool shaped) {
  TreePlan p;
  const int64_t columns = (int64_t)(n_heads / kv.n_kv_heads) * max_nodes;
  const bool e4m3 = kv.dtype == EMOE_E4M3;
  p.wide = columns > (kv.head_dim >= 128 ? 16 : 32);
  p.tiles = p.wide ? 4 : columns <= 16 ? 1 : 2;
  p.blocks = (int)((columns + 16 * p.tiles - 1) / (16 * p.tiles));
  p.lines = kv.n_kv_heads * p.blocks;
  const int64_t span = (int64_t)window + max_nodes;
  const int64_t keys = window > 0 && span < max_keys ? span : max_keys;
  // A step of the wide kernel; a tile for each wavefront of the other.
  p.unit_keys = kTileKeys * (p.wide ? wide_step_tiles(kv.head_dim, e4m3) : kTreeWaves);
  const int64_t most_units = (keys / p.unit_keys + 2) * p.blocks;
  const int64_t outputs = (int64_t)trees * p.lines;
  const int places = kUnits * (p.wide ? wide_workgroups(kv.head_dim, e4m3) : kv.head_dim == 256 ? 1 : 2);
  constexpr int kManyOutputs = 1024, kManyKeys = 2048, kLaunchOutputs = 1 << 14, kLaunchTrees = 1024;
  const bool many = outputs >= kManyOutputs;
  const int few_keys = many ? kManyKeys : (p.wide ? 256 : 512) * (outputs >= kUnits && !shaped ? 2 : 1);
  const bool may_cut = keys > few_keys && kv.n_kv_heads <= (many ? places / 8 : places) && p.lines <= kLaunchOutputs;
  // A launch's units stay below 2^31, its threads below 2^32, its trees within the grid's
  // third axis; those of one that is cut within what a worker looks through and the join's
  // descriptors.
  p.trees_per_launch = (((int64_t)1 << 31) - 1 - 4 * kUnits) / most_units;
  const bool whole = !may_cut || p.trees_per_launch < 1;
  if (whole) p.trees_per_launch = trees < 65535 ? trees : 65535;
  else if (p.trees_per_launch > kLaunchTrees) p.trees_per_launch = kLaunchTrees;
  const int64_t most_outputs = whole ? (int64_t)1 << 23 : kLaunchOutputs;
  if (p.trees_per_launch > most_outputs / p.lines) p.trees_per_launch = most_outputs / p.lines;
  p.workers = whole ? 0 : places / kv.n_kv_heads;
  // How much longer than equal runs the parts may be: 40 trees over 8 bits within 1% of 163
  // us from 4 to 40.
  p.slack = p.wide ? 12 : 6;
  p.part_floats = 16 * p.tiles * (2 + kv.head_dim);
  // Threads to an item of the join: 1 and 4 of them 159 and 177 us with 640 outputs (40 trees
  // over 8 bits), 100.6 and 97.3 with 8.
  p.stripes = outputs * 16 * p.tiles * (kv.head_dim / 4) / 256 < 1024 ? 4 : 1;
  // What a call with fewer keys (a window, a short table), or without shaped scores, takes is
  // no more than this.
  p.most_parts = may_cut ? 2 * (int64_t)(places / kv.n_kv_heads) * kv.n_kv_heads : 0;
  p.most_shared = !may_cut ? 0 : outputs < kLaunchOutputs ? outputs : kLaunchOutputs;
  return p;
}

size_t shared_bytes(const TreePlan& p) { return ((size_t)p.most_shared * 12 + 15) / 16 * 16; }

}  // namespace

extern "C" {

size_t emoe_paged_tree_attention_workspace_bytes(const emoe_paged_kv* kv, int32_t trees,
                                                 int32_t n_heads, int32_t max_keys,
                                                 int32_t max_nodes) {
  if (check_kv(kv) || trees < 0 || n_heads < 1 || n_heads % kv->n_kv_heads || max_keys < 0 ||
      max_keys > kMostKeys || n_heads > kMostHeads || max_nodes < 1 || max_nodes > EMOE_MAX_NODES ||
      (int64_t)(n_heads / kv->n_kv_heads) * max_nodes > kMostColumns)
    return 0;
  const TreePlan p = tree_plan(*kv, trees, n_heads, max_keys, max_nodes, 0, true);
  return 16 + shared_bytes(p) + (size_t)p.most_parts * p.part_floats * 4;
}

int32_t emoe_paged_tree_attention(const emoe_paged_kv* kv, const emoe_paged_tree_args* args,
                                  void* workspace, size_t workspace_bytes, hipStream_t stream) {
  int32_t st = check_kv(kv);
  if (st) return st;
  if (!args) return report_error(EMOE_EINVAL, "args is NULL");
  const emoe_paged_tree_args& A = *args;
  if ((st = check_io(*kv, A.dtype, A.page_table, A.n_seqs, A.table_width, A.table_stride))) return st;
  if (A.rows < 0 || A.trees < 0 || A.max_keys < 0 || A.window < 0)
    return report_error(EMOE_EINVAL, "negative rows, trees, max_keys or window (%d, %d, %d, %d)", A.rows,
                        A.trees, A.max_keys, A.window);
  if (A.max_nodes < 1 || A.max_nodes > EMOE_MAX_NODES)
    return report_error(EMOE_ESHAPE, "max_nodes %d: need 1 to %d", A.max_nodes, EMOE_MAX_NODES);
  if (A.n_heads < 1 || A.n_heads % kv->n_kv_heads)
    return report_error(EMOE_ESHAPE, "n_heads %d is no multiple of n_kv_heads %d", A.n_heads,
                        kv->n_kv_heads);
  if (A.max_keys > kMostKeys || A.n_heads > kMostHeads)
    return report_error(EMOE_ESHAPE, "max_keys %d or n_heads %d: need at most 2^30 and 2^20", A.max_keys,
                        A.n_heads);
  if ((int64_t)(A.n_heads / kv->n_kv_heads) * A.max_nodes > kMostColumns)
    return report_error(EMOE_ESHAPE, "%d query heads to a key head, of %d nodes: need a product of at most 2^20",
                        A.n_heads / kv->n_kv_heads, A.max_nodes);
  if (!A.starts && A.rows != (int64_t)A.trees * A.max_nodes)
    return report_error(EMOE_ESHAPE, "%d rows without starts: need %d trees of %d nodes", A.rows, A.trees,
                        A.max_nodes);
  if (!std::isfinite(A.scale * 1.4426950408889634f))  // as the kernel takes it
    return report_error(EMOE_EINVAL, "scale %g is not finite, or near the largest number", A.scale);
  if (!(A.cap == 0.f || (A.cap >= 0x1p-60f && A.cap <= 0x1p60f)))
    return report_error(EMOE_EINVAL, "cap %g: need 0 (none) or 2^-60 to 2^60", A.cap);
  if (A.rows == 0 || A.trees == 0) return EMOE_OK;
  const int64_t qw = (int64_t)A.n_heads * kv->head_dim;
  if ((st = check_rows("q", A.q, A.q_stride, A.rows, qw))) return st;
  if ((st = check_rows("out", A.out, A.out_stride, A.rows, qw))) return st;
  if (!A.lengths) return report_error(EMOE_EINVAL, "lengths is NULL");
  const size_t bytes =
      emoe_paged_tree_attention_workspace_bytes(kv, A.trees, A.n_heads, A.max_keys, A.max_nodes);
  if (!workspace || workspace_bytes < bytes)
    return report_error(EMOE_EINVAL, "workspace of %zu bytes < %zu needed", workspace ? workspace_bytes : 0,
                        bytes);
  if (!aligned16(workspace)) return report_error(EMOE_EINVAL, "workspace: need 16-byte alignment");
  const int64_t held = (int64_t)A.table_width * kv->page_size;  // no more keys than the table holds
  const TreePlan plan = tree_plan(*kv, A.trees, A.n_heads, held < A.max_keys ? held : A.max_keys,
                                  A.max_nodes, A.window, A.cap > 0.f || A.slopes);
  TreeArg a;
  a.kv = view_of(*kv);
  a.q = static_cast<const uint16_t*>(A.q);
  a.out = static_cast<uint16_t*>(A.out);
  a.lse = A.lse;
  a.lengths = A.lengths;
  a.starts = A.starts;
  a.seqs = A.seqs;
  a.tree = A.tree;
  a.slopes = A.slopes;
  a.table = A.page_table;
  a.heads_of = static_cast<int32_t*>(workspace);
  a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + shared_bytes(plan));
  a.q_stride = A.q_stride;
  a.out_stride = A.out_stride;
  a.table_stride = A.table_stride;
  a.scale = A.scale;
  a.cap = A.cap;
  a.rows = A.rows;
  a.n_heads = A.n_heads;
  a.group = A.n_heads / kv->n_kv_heads;
  a.blocks = plan.blocks;
  a.n_seqs = A.n_seqs;
  a.table_width = A.table_width;
  a.max_keys = A.max_keys;
  a.max_nodes = A.max_nodes;
  a.window = A.window;
  a.workers = plan.workers;
  a.slack = plan.slack;
  a.unit_keys = plan.unit_keys;
  a.unit_log2 = __builtin_ctz((unsigned)a.unit_keys);
  a.part_floats = plan.part_floats;
  for (int64_t t0 = 0; t0 < A.trees; t0 += plan.trees_per_launch) {
    a.tree0 = (int32_t)t0;
    a.trees = (int32_t)(A.trees - t0 < plan.trees_per_launch ? A.trees - t0 : plan.trees_per_launch);
    if (A.dtype == EMOE_BF16) launch_tree_bf16(a, plan, kv->head_dim, kv->dtype == EMOE_E4M3, stream);
    else launch_tree_fp16(a, plan, kv->head_dim, kv->dtype == EMOE_E4M3, stream);
    if ((st = launched("paged_tree_kernel"))) return st;
  }
  return EMOE_OK;
}

}  // extern "C"
