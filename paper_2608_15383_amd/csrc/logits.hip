// Between the logits and the next token (exactmoe_serving.h): penalties for
// repeated tokens, biases, grammar masks and the greedy choice.
#include "serving.h"

using namespace emoe;

namespace {

constexpr int kThreads = 256;
constexpr int kTickets = EMOE_SERVING_TICKET_BYTES / 4;

struct LogitsArg {
  const void* logits;
  void* out;
  int32_t* next_token;
  const int32_t *history, *history_lengths, *prompt_lengths;
  const float *repetition, *presence, *frequency;
  const int32_t* bias_ids;
  const float* bias_values;
  const int32_t* bias_counts;
  const uint32_t* mask;
  const int32_t* mask_rows;
  uint32_t* tickets;
  uint64_t* best;  // [row of the launch][chunk]
  int64_t logits_stride, out_stride, history_stride, bias_stride, mask_stride;
  int32_t row0, vocab, history_width, bias_width, n_masks, chunks;
};

struct F32 {
  static constexpr int kPer = 4;  // elements of a 16-byte chunk
  __device__ static __forceinline__ void up(const uint4& c, float (&v)[4]) {
    v[0] = __uint_as_float(c.x);
    v[1] = __uint_as_float(c.y);
    v[2] = __uint_as_float(c.z);
    v[3] = __uint_as_float(c.w);
  }
  __device__ static __forceinline__ uint4 down(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                      __float_as_uint(v[3]));
  }
  typedef uint32_t Raw;
  __device__ static __forceinline__ float up1(Raw r) { return __uint_as_float(r); }
  __device__ static __forceinline__ Raw down1(float x) { return __float_as_uint(x); }
};
template <class T>
struct Half {
  static constexpr int kPer = 8;
  __device__ static __forceinline__ void up(const uint4& c, float (&v)[8]) { up8<T>(c, v); }
  __device__ static __forceinline__ uint4 down(const float (&v)[8]) { return down8<T>(v); }
  typedef uint16_t Raw;
  __device__ static __forceinline__ float up1(Raw r) { return T::up(r); }
  __device__ static __forceinline__ Raw down1(float x) { return (Raw)T::down(x); }
};

// A value and its index as one word whose order is (value ascending, index
// descending); 0 for what is never chosen (NaN and -inf).
__device__ __forceinline__ uint64_t choice(float x, int v) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(x + 0.0f);  // -0 ties with +0
  const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((uint64_t)o << 32) | (uint32_t)~v;
}
__device__ __forceinline__ int chosen(uint64_t c) { return c ? (int)~(uint32_t)c : -1; }
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

__device__ __forceinline__ uint64_t wave_max(uint64_t c) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) c = max64(c, (uint64_t)__shfl_xor((unsigned long long)c, o));
  return c;
}

// A workgroup takes one chunk of one row: its logits are on their way while
// the row's history (and biases) is counted into words of LDS, one per token
// id of the chunk (bit 31: in the prompt; low bits: times generated), then one
// pass applies everything, writes the row and keeps the best.  Counting again
// for every chunk costs L2 reads of the history, but needs no table in memory
// as long as the vocabulary, which would have to be cleared and read as well.
// The row's last workgroup to finish (a ticket in the workspace) takes the
// best of its chunks' best.  Rows start at any element: the chunks of 16 bytes
// are loaded unaligned.
template <class F, int kLoads, bool kBias>
__global__ __launch_bounds__(kThreads) void process_logits_kernel(LogitsArg a) {
#pragma clang fp contract(off)
  constexpr int kPer = F::kPer;
  constexpr int kChunk = kThreads * kPer * kLoads;
  typedef typename F::Raw Raw;
  __shared__ __attribute__((aligned(16))) uint32_t seen[kChunk];
  __shared__ __attribute__((aligned(16))) int32_t bias[kBias ? kChunk : 4];
  __shared__ uint64_t red[kThreads / 64];
  __shared__ int last;
  const int tid = threadIdx.x;
  const int lr = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int row = a.row0 + lr, c0 = chunk * kChunk;
  const int V = a.vocab;
  const Raw* src = static_cast<const Raw*>(a.logits) + row * a.logits_stride;
  uint4 raw[kLoads];
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int v = c0 + (u * kThreads + tid) * kPer;
    if (v + kPer <= V) {
      __builtin_memcpy(&raw[u], src + v, 16);
    } else {
      Raw e[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) e[i] = v + i < V ? src[v + i] : Raw(0);
      __builtin_memcpy(&raw[u], e, 16);
    }
  }
  const float rep = a.repetition ? a.repetition[row] : 1.f;
  const float pres = a.presence ? a.presence[row] : 0.f;
  const float freq = a.frequency ? a.frequency[row] : 0.f;
  const bool count = a.history && !(rep == 1.f && pres == 0.f && freq == 0.f);
  if (count) {
#pragma unroll
    for (int u = 0; u < kChunk / (4 * kThreads); ++u)
      reinterpret_cast<uint4*>(seen)[u * kThreads + tid] = make_uint4(0, 0, 0, 0);
  }
  if constexpr (kBias) {
#pragma unroll
    for (int u = 0; u < kChunk / (4 * kThreads); ++u)
      reinterpret_cast<uint4*>(bias)[u * kThreads + tid] = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  if (count) {
    int n = a.history_width;
    if (a.history_lengths) n = max(0, min(n, a.history_lengths[row]));
    const int prompt = a.prompt_lengths ? a.prompt_lengths[row] : 0;
    const int32_t* h = a.history + row * a.history_stride;
    auto add = [&](int i, int id) {
      const uint32_t at = (uint32_t)id - (uint32_t)c0;
      if (at < (uint32_t)kChunk && id < V) {
        if (i < prompt) atomicOr(&seen[at], 0x80000000u);
        else atomicAdd(&seen[at], 1u);
      }
    };
    for (int i = 4 * tid; i < n; i += 4 * kThreads) {
      if (i + 4 <= n) {
        int id[4];
        __builtin_memcpy(id, h + i, 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) add(i + k, id[k]);
      } else {
        for (int k = i; k < n; ++k) add(k, h[k]);
      }
    }
  }
  if constexpr (kBias) {
    int n = a.bias_width;
    if (a.bias_counts) n = max(0, min(n, a.bias_counts[row]));
    const int32_t* ids = a.bias_ids + row * a.bias_stride;
    for (int i = tid; i < n; i += kThreads) {
      const int id = ids[i];
      const uint32_t at = (uint32_t)id - (uint32_t)c0;
      if (at < (uint32_t)kChunk && id < V) atomicMax(&bias[at], i + 1);  // the later entry counts
    }
  }
  __syncthreads();
  const uint32_t* mask = nullptr;
  if (a.mask) {
    const int m = a.mask_rows ? a.mask_rows[row] : row;
    if ((uint32_t)m < (uint32_t)a.n_masks) mask = a.mask + m * a.mask_stride;
  }
  const float* bias_values = kBias ? a.bias_values + row * a.bias_stride : nullptr;
  Raw* dst = static_cast<Raw*>(a.out) + row * a.out_stride;
  uint64_t best = 0;
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int at = (u * kThreads + tid) * kPer, v = c0 + at;
    if (v >= V) break;
    float x[kPer];
    F::up(raw[u], x);
    const uint32_t bits = mask ? mask[v >> 5] >> (v & 31) : ~0u;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (count) {
        const uint32_t w = seen[at + i];
        if (w) {
          x[i] = x[i] > 0.f ? x[i] / rep : x[i] * rep;
          const uint32_t c = w & 0x7fffffffu;
          if (c) {
            const float f = freq * (float)c;
            x[i] = x[i] - f;
            x[i] = x[i] - pres;
          }
        }
      }
      if constexpr (kBias) {
        const int b = bias[at + i];
        if (b) x[i] = x[i] + bias_values[b - 1];
      }
      if (!((bits >> i) & 1)) x[i] = -INFINITY;
      if (v + i < V) best = max64(best, choice(x[i], v + i));
    }
    const uint4 o = F::down(x);
    if (v + kPer <= V) {
      __builtin_memcpy(dst + v, &o, 16);
    } else {
      for (int i = 0; v + i < V; ++i) dst[v + i] = F::down1(x[i]);
    }
  }
  if (!a.next_token) return;
  best = wave_max(best);
  if ((tid & 63) == 0) red[tid >> 6] = best;
  __syncthreads();
  if (tid == 0) {
    best = max64(max64(red[0], red[1]), max64(red[2], red[3]));
    last = 0;
    if (a.chunks == 1) {
      a.next_token[row] = chosen(best);
    } else {
      __hip_atomic_store(&a.best[(int64_t)lr * a.chunks + chunk], best, __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
      wait_memory();
      last = __hip_atomic_fetch_add(&a.tickets[lr], 1u, __ATOMIC_RELAXED,
                                    __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.chunks - 1;
      wait_memory();
    }
  }
  if (a.chunks == 1) return;
  __syncthreads();
  if (!last || tid >= 64) return;
  best = 0;
  for (int i = tid; i < a.chunks; i += 64)
    best = max64(best, __hip_atomic_load(&a.best[(int64_t)lr * a.chunks + i], __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT));
  best = wave_max(best);
  if (tid == 0) {
    a.next_token[row] = chosen(best);
    st_u32<true>(&a.tickets[lr], 0);
  }
}

template <class F, int kLoads>
void launch_logits(const LogitsArg& a, unsigned blocks, hipStream_t stream) {
  if (a.bias_ids)
    hipLaunchKernelGGL((process_logits_kernel<F, kLoads, true>), dim3(blocks), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((process_logits_kernel<F, kLoads, false>), dim3(blocks), dim3(kThreads), 0, stream, a);
}

template <class F>
void launch_type(const LogitsArg& a, int loads, unsigned blocks, hipStream_t stream) {
  if (loads == 1) launch_logits<F, 1>(a, blocks, stream);
  else launch_logits<F, 4>(a, blocks, stream);
}

int chunks_of(int32_t vocab, int per, int loads) {
  const int64_t c = (int64_t)kThreads * per * loads;
  return (int)((vocab + c - 1) / c);
}

}  // namespace

extern "C" {

size_t emoe_process_logits_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 0 || vocab < 1) return 0;
  const size_t held = rows < kTickets ? rows : kTickets;  // rows of one launch
  return EMOE_SERVING_TICKET_BYTES + held * (size_t)chunks_of(vocab, F32::kPer, 1) * 8;
}

int32_t emoe_process_logits(const emoe_logits_args* args, void* workspace, size_t workspace_bytes,
                            hipStream_t stream) {
  if (!args) return report_error(EMOE_EINVAL, "args is NULL");
  const emoe_logits_args& A = *args;
  if (A.dtype != EMOE_F32 && A.dtype != EMOE_BF16 && A.dtype != EMOE_F16)
    return report_error(EMOE_EINVAL, "type %d: need f32, bf16 or fp16", A.dtype);
  if (A.rows < 0 || A.vocab < 1)
    return report_error(EMOE_ESHAPE, "rows %d, vocab %d", A.rows, A.vocab);
  if (A.vocab > (1 << 30)) return report_error(EMOE_ESHAPE, "vocab %d above 2^30", A.vocab);
  if (A.history_width < 0 || A.bias_width < 0 || A.n_masks < 0)
    return report_error(EMOE_EINVAL, "negative history_width, bias_width or n_masks");
  if (A.rows == 0) return EMOE_OK;
  if (!A.logits || !A.out) return report_error(EMOE_EINVAL, "NULL logits or out");
  const uintptr_t item = A.dtype == EMOE_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(A.logits) % item || reinterpret_cast<uintptr_t>(A.out) % item)
    return report_error(EMOE_EINVAL, "logits or out not aligned to their elements");
  const bool many = A.rows > 1;
  if (many && (A.logits_stride < A.vocab || A.out_stride < A.vocab))
    return report_error(EMOE_EINVAL, "logits or out: row stride below vocab %d", A.vocab);
  if (A.history && many && A.history_stride < A.history_width)
    return report_error(EMOE_EINVAL, "history_stride below history_width %d", A.history_width);
  if (!A.history && (A.repetition || A.presence || A.frequency))
    return report_error(EMOE_EINVAL, "penalties without a history");
  if (!A.bias_ids != !A.bias_values)
    return report_error(EMOE_EINVAL, "one of bias_ids and bias_values is NULL");
  if (A.bias_ids && many && A.bias_stride < A.bias_width)
    return report_error(EMOE_EINVAL, "bias_stride below bias_width %d", A.bias_width);
  if (A.mask) {
    if (A.n_masks > 1 && A.mask_stride < (A.vocab + (int64_t)31) / 32)
      return report_error(EMOE_EINVAL, "mask_stride %lld below ceil(vocab / 32)", (long long)A.mask_stride);
    if (!A.mask_rows && A.n_masks < A.rows)
      return report_error(EMOE_EINVAL, "%d masks for %d rows", A.n_masks, A.rows);
  } else if (A.mask_rows) {
    return report_error(EMOE_EINVAL, "mask_rows without a mask");
  }
  const int per = A.dtype == EMOE_F32 ? 4 : 8;
  const int loads = (int64_t)A.rows * chunks_of(A.vocab, per, 4) >= 512 ? 4 : 1;
  const int chunks = chunks_of(A.vocab, per, loads);
  if (A.next_token) {
    const size_t need = emoe_process_logits_workspace_bytes(A.rows, A.vocab);
    if (!workspace || workspace_bytes < need)
      return report_error(EMOE_EINVAL, "workspace of %zu bytes < %zu needed",
                          workspace ? workspace_bytes : 0, need);
    if (!aligned16(workspace)) return report_error(EMOE_EINVAL, "workspace: need 16-byte alignment");
  }
  LogitsArg a;
  a.logits = A.logits;
  a.out = A.out;
  a.next_token = A.next_token;
  a.history = A.history;
  a.history_lengths = A.history_lengths;
  a.prompt_lengths = A.prompt_lengths;
  a.repetition = A.repetition;
  a.presence = A.presence;
  a.frequency = A.frequency;
  a.bias_ids = A.bias_width > 0 ? A.bias_ids : nullptr;
  a.bias_values = A.bias_values;
  a.bias_counts = A.bias_counts;
  a.mask = A.mask;
  a.mask_rows = A.mask_rows;
  a.tickets = static_cast<uint32_t*>(workspace);
  a.best = reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(workspace) + EMOE_SERVING_TICKET_BYTES);
  if (!A.next_token) a.tickets = nullptr, a.best = nullptr;
  a.logits_stride = A.logits_stride;
  a.out_stride = A.out_stride;
  a.history_stride = A.history_stride;
  a.bias_stride = A.bias_stride;
  a.mask_stride = A.mask_stride;
  a.vocab = A.vocab;
  a.history_width = A.history_width;
  a.bias_width = A.bias_width;
  a.n_masks = A.n_masks;
  a.chunks = chunks;
  // Rows of one launch: a ticket each, and a grid below 2^31 workgroups.
  int64_t step = ((int64_t)1 << 30) / chunks;
  if (step > kTickets) step = kTickets;
  for (int64_t r0 = 0; r0 < A.rows; r0 += step) {
    a.row0 = (int32_t)r0;
    const int64_t n = A.rows - r0 < step ? A.rows - r0 : step;
    const unsigned blocks = (unsigned)(n * chunks);
    if (A.dtype == EMOE_F32) launch_type<F32>(a, loads, blocks, stream);
    else if (A.dtype == EMOE_BF16) launch_type<Half<Bf16>>(a, loads, blocks, stream);
    else launch_type<Half<Fp16>>(a, loads, blocks, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
      return report_error(EMOE_EHIP, "process_logits_kernel launch: %s", hipGetErrorString(e));
  }
  return EMOE_OK;
}

}  // extern "C"
