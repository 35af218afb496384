// The paged key-value cache (exactmoe_serving.h): append with the rotary
// positions on the way, and the attention of one new token per row.
#include <cmath>

#include "device_rope.h"
#include "serving.h"

using namespace emoe;

namespace {

constexpr int kThreads = 256;

// What the kernels need of the cache; strides in bytes.
struct KvView {
  uint8_t *k, *v;
  const float *k_scale, *v_scale;
  int64_t page_bytes;
  int32_t slot_bytes, head_bytes;
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
  int32_t tokens, n_heads, n_seqs, table_width, rotary_dim;
};

// One item is a pair of 16-byte chunks (16 dimensions) of one head of q, k or
// v.  Halves: chunk i of the first half of the rotated dimensions and the one
// that it turns with; interleaved or not rotated: two neighbours.  A workgroup
// takes kTok tokens, forms their angles' cosines and sines once (fp64, shared
// by all heads) and then walks over their items; blockIdx.y splits the items
// of small calls.  Bound by HBM: every value is read and written once.
constexpr int kTok = 4;
template <class T, bool kE4M3, bool kInter, int kDh>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(AppendArg a) {
  __shared__ float2 cs[kTok][kDh / 2];
  __shared__ int64_t slot_at[kTok];  // byte offset of the token's slot, -1: none
  __shared__ int live[kTok];
  constexpr int kPieces = kDh / 16;
  const int t0 = blockIdx.x * kTok;
  const int half = a.rotary_dim / 2;
  if (threadIdx.x < kTok) {
    const int t = t0 + threadIdx.x;
    int64_t at = -1;
    int ok = 0;
    if (t < a.tokens) {
      const int p = a.positions[t], s = a.seqs ? a.seqs[t] : t;
      ok = p >= 0 && (uint32_t)s < (uint32_t)a.n_seqs;
      const int col = p >> a.kv.page_log2;
      if (ok && col < a.table_width) {
        const int page = a.table[(int64_t)s * a.table_stride + col];
        if ((uint32_t)page < (uint32_t)a.kv.n_pages)
          at = page * a.kv.page_bytes +
               (int64_t)(p & ((1 << a.kv.page_log2) - 1)) * a.kv.slot_bytes;
      }
    }
    slot_at[threadIdx.x] = at;
    live[threadIdx.x] = ok;
  }
  for (int x = threadIdx.x; x < kTok * half; x += kThreads) {
    const int tt = x / half, i = x % half;
    if (t0 + tt < a.tokens) {
      float2 w;
      rope_cos_sin((double)a.positions[t0 + tt] * a.inv_freq[i], w.x, w.y);
      cs[tt][i] = w;
    }
  }
  __syncthreads();
  const int heads = (a.q ? a.n_heads : 0) + 2 * a.kv.n_kv_heads;
  const int per_tok = heads * kPieces;
  const int n_items = min(kTok, a.tokens - t0) * per_tok;
  for (int x = blockIdx.y * kThreads + threadIdx.x; x < n_items; x += gridDim.y * kThreads) {
    const int tt = x / per_tok, j = x % per_tok;
    const int64_t t = t0 + tt;
    int h = j / kPieces;
    const int pc = j % kPieces;
    const int q_heads = a.q ? a.n_heads : 0;
    const int kind = h < q_heads ? 0 : (h < q_heads + a.kv.n_kv_heads ? 1 : 2);
    h -= kind == 0 ? 0 : (kind == 1 ? q_heads : q_heads + a.kv.n_kv_heads);
    if (!live[tt] || (kind != 0 && slot_at[tt] < 0)) continue;
    // The two chunks (8 dimensions each) and, when they turn, their first pair.
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
    up8<T>(row[c0], x0);
    up8<T>(row[c1], x1);
    if (turns) {
      if constexpr (kInter) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 w0 = cs[tt][8 * pc + i], w1 = cs[tt][8 * pc + 4 + i];
          const float a0 = x0[2 * i], b0 = x0[2 * i + 1], a1 = x1[2 * i], b1 = x1[2 * i + 1];
          x0[2 * i] = fmaf(a0, w0.x, -(b0 * w0.y));
          x0[2 * i + 1] = fmaf(a0, w0.y, b0 * w0.x);
          x1[2 * i] = fmaf(a1, w1.x, -(b1 * w1.y));
          x1[2 * i + 1] = fmaf(a1, w1.y, b1 * w1.x);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 w = cs[tt][8 * pc + i];
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
      uint8_t* dst = (kind == 1 ? a.kv.k : a.kv.v) + slot_at[tt] + (int64_t)h * a.kv.head_bytes;
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
  int64_t q_stride, out_stride, table_stride;
  float scale;
  int32_t rows, n_heads, n_seqs, table_width, max_keys, window;
};

template <class T, bool kE4M3>
__device__ __forceinline__ float cache_value(const uint8_t* p, int i) {
  if constexpr (kE4M3) return __builtin_amdgcn_cvt_f32_fp8((int)p[i], 0);
  else return T::up(reinterpret_cast<const uint16_t*>(p)[i]);
}

// One workgroup per (query head, row): tiles of 256 keys, a thread per key for
// the scores and a thread per (dimension, key stripe) for the output, with the
// running maximum and sum of the softmax.
template <class T, bool kE4M3, int kDh>
__global__ __launch_bounds__(kThreads) void paged_attention_kernel(AttendArg a) {
  constexpr int kStripes = kThreads / kDh;
  __shared__ float qs[kDh], ps[kThreads], red[4], part[kStripes][kDh];
  __shared__ int64_t at[kThreads];
  const int h = blockIdx.x % a.n_heads, r = blockIdx.x / a.n_heads, tid = threadIdx.x;
  const int g = h / (a.n_heads / a.kv.n_kv_heads);
  const int s = a.seqs ? a.seqs[r] : r;
  int n = 0;
  if ((uint32_t)s < (uint32_t)a.n_seqs) {
    n = max(0, min(a.lengths[r], a.max_keys));
    n = (int)min((int64_t)n, (int64_t)a.table_width << a.kv.page_log2);
  }
  const int first = a.window > 0 ? max(0, n - a.window) : 0;
  if (tid < kDh) qs[tid] = T::up(a.q[r * a.q_stride + (int64_t)h * kDh + tid]);
  const float scale = a.scale * (kE4M3 && a.kv.k_scale ? a.kv.k_scale[g] : 1.0f);
  float m = -INFINITY, l = 0.f, acc = 0.f;
  const int dim = tid % kDh, stripe = tid / kDh;
  for (int base = first; base < n; base += kThreads) {
    const int j = base + tid;
    int64_t off = -1;
    float z = -INFINITY;
    __syncthreads();
    if (j < n) {
      const int page = a.table[(int64_t)s * a.table_stride + (j >> a.kv.page_log2)];
      if ((uint32_t)page < (uint32_t)a.kv.n_pages) {
        off = page * a.kv.page_bytes + (int64_t)(j & ((1 << a.kv.page_log2) - 1)) * a.kv.slot_bytes +
              (int64_t)g * a.kv.head_bytes;
        z = 0.f;
        for (int i = 0; i < kDh; ++i) z = fmaf(qs[i], cache_value<T, kE4M3>(a.kv.k + off, i), z);
        z *= scale;
      }
    }
    at[tid] = off;
    float mx = z;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    __syncthreads();
    const float m2 = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), m);
    const float ref = m2 == -INFINITY ? 0.f : m2;
    const float p = off >= 0 ? expf(z - ref) : 0.f;
    const float shrink = expf(m - ref);
    m = m2;
    ps[tid] = p;
    float sum = p;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o);
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = sum;
    __syncthreads();
    l = l * shrink + ((red[0] + red[1]) + (red[2] + red[3]));
    acc *= shrink;
    for (int i = stripe; i < min(kThreads, n - base); i += kStripes)
      if (at[i] >= 0) acc = fmaf(ps[i], cache_value<T, kE4M3>(a.kv.v + at[i], dim), acc);
  }
  part[stripe][dim] = acc;
  __syncthreads();
  if (tid < kDh) {
    float o = 0.f;
    for (int i = 0; i < kStripes; ++i) o += part[i][tid];
    o = l == 0.f ? 0.f : o / l;
    if (kE4M3 && a.kv.v_scale) o *= a.kv.v_scale[g];
    a.out[r * a.out_stride + (int64_t)h * kDh + tid] = (uint16_t)T::down(o);
  }
  if (tid == 0 && a.lse) a.lse[(int64_t)r * a.n_heads + h] = l == 0.f ? -INFINITY : m + logf(l);
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
void launch_attend(const AttendArg& a, int head_dim, hipStream_t stream) {
  const dim3 grid((unsigned)(a.n_heads * a.rows));
  if (head_dim == 64)
    hipLaunchKernelGGL((paged_attention_kernel<T, kE4M3, 64>), grid, dim3(kThreads), 0, stream, a);
  else if (head_dim == 128)
    hipLaunchKernelGGL((paged_attention_kernel<T, kE4M3, 128>), grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((paged_attention_kernel<T, kE4M3, 256>), grid, dim3(kThreads), 0, stream, a);
}

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
  if (A.q && A.n_heads < 1) return report_error(EMOE_ESHAPE, "n_heads %d", A.n_heads);
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
  a.tokens = A.tokens;
  a.n_heads = A.n_heads;
  a.n_seqs = A.n_seqs;
  a.table_width = A.table_width;
  a.rotary_dim = A.rotary_dim;
  const int64_t heads = (A.q ? A.n_heads : 0) + 2 * (int64_t)kv->n_kv_heads;
  const int64_t items = (int64_t)(A.tokens < kTok ? A.tokens : kTok) * heads * (dh / 16);
  if (items >= (int64_t)1 << 31) return report_error(EMOE_ESHAPE, "%lld heads", (long long)heads);
  const unsigned gx = (unsigned)((A.tokens + (int64_t)kTok - 1) / kTok);
  // Small calls: an item per thread.
  unsigned gy = 1;
  while (gx * gy < 512 && (int64_t)gy * kThreads < items) ++gy;
  const dim3 grid(gx, gy);
  const bool e4m3 = kv->dtype == EMOE_E4M3, inter = A.interleaved != 0;
  if (A.dtype == EMOE_BF16) {
    if (e4m3) launch_append<Bf16, true>(a, kv->head_dim, inter, grid, stream);
    else launch_append<Bf16, false>(a, kv->head_dim, inter, grid, stream);
  } else {
    if (e4m3) launch_append<Fp16, true>(a, kv->head_dim, inter, grid, stream);
    else launch_append<Fp16, false>(a, kv->head_dim, inter, grid, stream);
  }
  return launched("paged_append_kernel");
}

size_t emoe_paged_attention_workspace_bytes(const emoe_paged_kv* kv, int32_t rows, int32_t n_heads,
                                            int32_t max_keys) {
  if (check_kv(kv) || rows < 0 || n_heads < 1 || n_heads % kv->n_kv_heads || max_keys < 0) return 0;
  return EMOE_SERVING_TICKET_BYTES;
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
  if (!std::isfinite(A.scale)) return report_error(EMOE_EINVAL, "scale is not finite");
  if (A.rows == 0) return EMOE_OK;
  if ((int64_t)A.rows * A.n_heads >= (int64_t)1 << 30)
    return report_error(EMOE_ESHAPE, "%d rows of %d heads", A.rows, A.n_heads);
  const int64_t qw = (int64_t)A.n_heads * kv->head_dim;
  if ((st = check_rows("q", A.q, A.q_stride, A.rows, qw))) return st;
  if ((st = check_rows("out", A.out, A.out_stride, A.rows, qw))) return st;
  if (!A.lengths) return report_error(EMOE_EINVAL, "lengths is NULL");
  const size_t need = emoe_paged_attention_workspace_bytes(kv, A.rows, A.n_heads, A.max_keys);
  if (!workspace || workspace_bytes < need)
    return report_error(EMOE_EINVAL, "workspace of %zu bytes < %zu needed", workspace ? workspace_bytes : 0,
                        need);
  if (!aligned16(workspace)) return report_error(EMOE_EINVAL, "workspace: need 16-byte alignment");
  AttendArg a;
  a.kv = view_of(*kv);
  a.q = static_cast<const uint16_t*>(A.q);
  a.out = static_cast<uint16_t*>(A.out);
  a.lse = A.lse;
  a.lengths = A.lengths;
  a.seqs = A.seqs;
  a.table = A.page_table;
  a.q_stride = A.q_stride;
  a.out_stride = A.out_stride;
  a.table_stride = A.table_stride;
  a.scale = A.scale;
  a.rows = A.rows;
  a.n_heads = A.n_heads;
  a.n_seqs = A.n_seqs;
  a.table_width = A.table_width;
  a.max_keys = A.max_keys;
  a.window = A.window;
  const bool e4m3 = kv->dtype == EMOE_E4M3;
  if (A.dtype == EMOE_BF16) {
    if (e4m3) launch_attend<Bf16, true>(a, kv->head_dim, stream);
    else launch_attend<Bf16, false>(a, kv->head_dim, stream);
  } else {
    if (e4m3) launch_attend<Fp16, true>(a, kv->head_dim, stream);
    else launch_attend<Fp16, false>(a, kv->head_dim, stream);
  }
  return launched("paged_attention_kernel");
}

}  // extern "C"
