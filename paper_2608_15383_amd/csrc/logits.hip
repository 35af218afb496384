// Between the logits and the next token (exactmoe_serving.h): penalties for
// repeated tokens, biases, grammar masks and the greedy choice.
#include "serving.h"

using namespace emoe;

namespace {

constexpr int kMaxRows = 4096;  // rows of one launch
constexpr int kLongHistory = 6144;
constexpr uint32_t kBiasIndices = 1u << 23;  // bits of the smallest normal number

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
  uint32_t* tickets;  // [row of the launch], a line each: workgroups that have started
  uint64_t* best;     // [row of the launch][chunk]: the chunks' best choices, handed over
  int64_t logits_stride, out_stride, history_stride, bias_stride, mask_stride;
  int32_t row0, vocab, history_width, bias_width, n_masks, chunks;
};

// The element types: a 16-byte chunk holds kPer elements in four words.
struct F32 {
  static constexpr int kPer = 4;
  typedef uint32_t Raw;
  static constexpr uint32_t kLowest = 0xff800000u;  // -infinity
  __device__ static __forceinline__ float up(Raw r) { return __uint_as_float(r); }
  __device__ static __forceinline__ Raw down(float x) { return __float_as_uint(x); }
};
template <class T>
struct Half {
  static constexpr int kPer = 8;
  typedef uint16_t Raw;
  static constexpr uint32_t kLowest = T::kType == EMOE_BF16 ? 0xff80u : 0xfc00u;
  __device__ static __forceinline__ float up(Raw r) { return T::up(r); }
  __device__ static __forceinline__ Raw down(float x) { return (Raw)T::down(x); }
};

// Element i of a chunk, read and replaced by selects of values: an index into
// the words, or a conditional that chooses one of them as an lvalue, would put
// the chunk in memory.
__device__ __forceinline__ uint32_t pick(bool c, uint32_t a, uint32_t b) { return c ? a : b; }
template <class F>
__device__ __forceinline__ typename F::Raw element(const uint4& w, int i) {
  const int k = F::kPer == 4 ? i : i >> 1;
  const uint32_t x = pick(k & 2, pick(k & 1, w.w, w.z), pick(k & 1, w.y, w.x));
  return (typename F::Raw)(F::kPer == 4 ? x : x >> (16 * (i & 1)));
}
template <class F>
__device__ __forceinline__ uint32_t with_element(uint32_t w, int i, typename F::Raw r) {
  if (F::kPer == 4) return r;
  return i & 1 ? (w & 0xffffu) | ((uint32_t)r << 16) : (w & 0xffff0000u) | r;
}
template <class F>
__device__ __forceinline__ void put(uint4& w, int i, typename F::Raw r) {
  const int k = F::kPer == 4 ? i : i >> 1;
  w.x = pick(k == 0, with_element<F>(w.x, i, r), w.x);
  w.y = pick(k == 1, with_element<F>(w.y, i, r), w.y);
  w.z = pick(k == 2, with_element<F>(w.z, i, r), w.z);
  w.w = pick(k == 3, with_element<F>(w.w, i, r), w.w);
}
// Word k of a chunk with the elements that a mask does not allow replaced by
// -infinity: each bit is spread over its element, then chooses bits.
template <class F>
__device__ __forceinline__ uint32_t masked(uint32_t w, uint32_t allowed, int k) {
  auto spread = [&](int i) { return (uint32_t)((int32_t)(allowed << (31 - i)) >> 31); };
  uint32_t keep, low;
  if (F::kPer == 4) {
    keep = spread(k);
    low = F::kLowest;
  } else {
    keep = (spread(2 * k) & 0xffffu) | (spread(2 * k + 1) & 0xffff0000u);
    low = F::kLowest | (F::kLowest << 16);
  }
  return (w & keep) | (low & ~keep);
}
// Ids i .. i + 3 of a history of `width` ids, -1 past its end.
__device__ __forceinline__ int4 load_ids(const int32_t* h, int i, int width) {
  int4 id = make_int4(-1, -1, -1, -1);
  if (i + 4 <= width) {
    __builtin_memcpy(&id, h + i, 16);
  } else {
    if (i < width) id.x = h[i];
    if (i + 1 < width) id.y = h[i + 1];
    if (i + 2 < width) id.z = h[i + 2];
  }
  return id;
}

// The chunk at src[v], of which elements from V on are read as 0.
template <class F>
__device__ __forceinline__ uint4 load_chunk(const typename F::Raw* src, int v, int V) {
  uint4 w = make_uint4(0, 0, 0, 0);
  if (v + F::kPer <= V) {
    __builtin_memcpy(&w, src + v, 16);
  } else {
#pragma unroll
    for (int i = 0; i < F::kPer; ++i)
      if (v + i < V) put<F>(w, i, src[v + i]);
  }
  return w;
}
template <class F>
__device__ __forceinline__ void store_chunk(typename F::Raw* dst, int v, int V, const uint4& w) {
  if (v + F::kPer <= V) {
    // Streaming: 256 rows of 131,072 bf16 logits take 32.7 us so, 40.7 with plain stores.
    typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));  // a 16-bit element at least
    __builtin_nontemporal_store(Words{w.x, w.y, w.z, w.w}, reinterpret_cast<Words*>(dst + v));
  } else {
#pragma unroll
    for (int i = 0; i < F::kPer; ++i)
      if (v + i < V) dst[v + i] = element<F>(w, i);
  }
}

// A value and its index as one word whose order is (value ascending, index
// descending); 0 for what is never chosen (NaN and -inf).
__device__ __forceinline__ uint64_t choice(float x, int v) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(x + 0.0f);  // -0 ties with +0
  const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((uint64_t)o << 32) | (uint32_t)~v;
}
// Hand-over between the workgroups of a row.  Each takes a ticket of the row when
// it starts, on the way with its loads; the one that starts last collects the
// row's choice.  A chunk's word is 0 until its workgroup stores its best, device-
// coherently, and 0 again when the collector has read it; kNoChoice stands for 0
// meanwhile.  The collector waits only for workgroups that run already and wait
// for nobody, so every wait ends, whatever else the device runs.  To count
// workgroups as they finish instead takes one trip to memory more, 0.6 us of the
// 5.8 that a row of 50,304 logits took so.  The wait is bounded (kSpinLimit polls,
// about a second) so that a launch ends over a workspace that was not zeroed, too.
// Its tokens are undefined: perhaps nobody starts last, or old words pass for
// choices, and tickets and words may stay nonzero for later calls.
constexpr uint64_t kNoChoice = 1;
constexpr int kSpinLimit = 1 << 19;
__device__ __forceinline__ int chosen(uint64_t c) { return c ? (int)~(uint32_t)c : -1; }
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

__device__ __forceinline__ uint64_t wave_max(uint64_t c) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) c = max64(c, (uint64_t)__shfl_xor((unsigned long long)c, o));
  return c;
}

// A workgroup takes one chunk of one row: its logits are on their way while
// the row's history (and biases) is counted into LDS, a counter per token id
// of the chunk.  Counting again for every chunk costs L2 reads of the
// history, but needs no table in memory as long as the vocabulary, which would
// have to be cleared and read as well.  Then one pass: the few touched elements
// are taken out of their registers one by one, the mask replaces words, and
// everything else goes from load to store as it came (a 16-bit logit is its
// own rounding); the greedy choice needs one comparison per chunk of 16 bytes
// unless that holds a new best.  One workgroup of the row takes the best of the
// chunks' best, which the others hand over.  Rows start at any
// element: the chunks of 16 bytes are loaded unaligned.
// Large calls are bound by HBM: 256 rows of 131,072 bf16 logits with masks and
// 1,000 ids take 32.3 us, 4.6 TB/s with the history read again per chunk.  Small
// ones are bound by trips to memory (logits and ids, then the hand-over): one row
// of 50,304 5.2 us; long histories by the LDS additions: 19 rows of 49,999 with
// 32,000 ids 15.2.
template <class F, int kThreads, int kLoads, bool kBias>
__global__ __launch_bounds__(kThreads) void process_logits_kernel(LogitsArg a) {
#pragma clang fp contract(off)
  constexpr int kPer = F::kPer;
  constexpr int kChunk = kThreads * kPer * kLoads;
  constexpr uint32_t kAll = (1u << kPer) - 1;
  typedef typename F::Raw Raw;
  // A counter per id: 16 bits where the history is short, so that twice the
  // workgroups fit a CU, else 32.  Low part: times generated; above it, that the
  // prompt has the id: a bit, or how often where both numbers fit their half of
  // 32 bits, so that one addition does.  64 words more take the additions of
  // the ids that lie in other chunks, which costs less than to skip them.
  constexpr bool kShort = kThreads == 256;
  static_assert(kLongHistory <= 0x8000, "15 bits hold a short history's counts");
  constexpr int kSeenWords = kShort ? kChunk / 2 : kChunk;
  __shared__ __attribute__((aligned(16))) uint32_t seen[kSeenWords + 64];
  __shared__ __attribute__((aligned(16))) int32_t bias[kBias ? kChunk : 4];
  __shared__ uint64_t red[kThreads / 64];
  const int tid = threadIdx.x;
  const int lr = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
  const int row = a.row0 + lr, c0 = chunk * kChunk;
  const int V = a.vocab;
  const Raw* src = static_cast<const Raw*>(a.logits) + row * a.logits_stride;
  // Everything that memory has to give is asked for first: the row's settings,
  // its logits, its mask and the beginning of its history (of the array's
  // width: how much of it counts is not known yet).
  const float rep = a.repetition ? a.repetition[row] : 1.f;
  const float pres = a.presence ? a.presence[row] : 0.f;
  const float freq = a.frequency ? a.frequency[row] : 0.f;
  int n_hist = a.history_lengths ? a.history_lengths[row] : a.history_width;
  const int prompt = a.prompt_lengths ? a.prompt_lengths[row] : 0;
  int n_bias = a.bias_counts ? a.bias_counts[row] : a.bias_width;
  const int mask_row = a.mask_rows ? a.mask_rows[row] : row;
  uint4 raw[kLoads];
  uint32_t allow[kLoads];
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int v = c0 + (u * kThreads + tid) * kPer;
    raw[u] = load_chunk<F>(src, v, V);
    allow[u] = kAll;
    if (a.mask && (uint32_t)mask_row < (uint32_t)a.n_masks && v < V)
      allow[u] = a.mask[mask_row * a.mask_stride + (v >> 5)] >> (v & 31) & kAll;
    if (v + kPer > V) allow[u] &= v < V ? (1u << (V - v)) - 1 : 0;
  }
  const int32_t* hist = a.history + row * a.history_stride;
  constexpr int kAhead = kShort ? 1 : 4;  // loads of four ids in flight per thread
  int4 ids[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    ids[k] = a.history ? load_ids(hist, 4 * (k * kThreads + tid), a.history_width)
                       : make_int4(-1, -1, -1, -1);
  int bias_id = -1;
  float bias_value = 0.f;
  if constexpr (kBias) {
    if (tid < a.bias_width) {
      bias_id = a.bias_ids[row * a.bias_stride + tid];
      bias_value = a.bias_values[row * a.bias_stride + tid];
    }
  }
  // After the loads, which return in order.
  const bool choose = a.next_token != nullptr;
  uint32_t* ticket = a.tickets + (int64_t)lr * kTicketStride;
  uint32_t order = 0;
  if (choose && a.chunks > 1 && tid == 0)
    order = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  n_hist = max(0, min(n_hist, a.history_width));
  n_bias = max(0, min(n_bias, a.bias_width));
  const bool count = a.history && !(rep == 1.f && pres == 0.f && freq == 0.f);
  const bool both = !kShort && a.history_width < 0x10000;
  const uint32_t made_bits = kShort ? 0x7fffu : both ? 0xffffu : 0x7fffffffu;
  if (count || kBias) {
    if (count)
      for (int i = tid; i < kSeenWords / 4; i += kThreads)
        reinterpret_cast<uint4*>(seen)[i] = make_uint4(0, 0, 0, 0);
    if constexpr (kBias)
      for (int i = tid; i < kChunk / 4; i += kThreads)
        reinterpret_cast<uint4*>(bias)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    if (count) {
      const uint32_t here = (uint32_t)min(kChunk, V - c0);
      auto add = [&](int i, int id) __attribute__((always_inline)) {
        const uint32_t at = (uint32_t)id - (uint32_t)c0;
        const bool hit = at < here && i < n_hist, old = i < prompt;
        if constexpr (kShort) {
          uint32_t* word = &seen[hit ? at >> 1 : kSeenWords + (tid & 63)];
          const int sh = 16 * (at & 1);
          atomicAdd(word, old ? 0u : 1u << sh);
          if (old) atomicOr(word, 0x8000u << sh);
        } else {
          uint32_t* word = &seen[hit ? at : kSeenWords + (tid & 63)];
          if (both) atomicAdd(word, old ? 0x10000u : 1u);
          else if (old) atomicOr(word, 0x80000000u);
          else atomicAdd(word, 1u);
        }
      };
      for (int i0 = 0; i0 < n_hist; i0 += 4 * kThreads * kAhead) {
        if (i0 > 0) {
#pragma unroll
          for (int k = 0; k < kAhead; ++k)
            ids[k] = load_ids(hist, i0 + 4 * (k * kThreads + tid), a.history_width);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int i = i0 + 4 * (k * kThreads + tid);
          add(i, ids[k].x);
          add(i + 1, ids[k].y);
          add(i + 2, ids[k].z);
          add(i + 3, ids[k].w);
        }
      }
    }
    if constexpr (kBias) {
      // The later of two entries of an id counts: the largest index stays in the
      // id's word, then gives way to the entry's value, whose bits cannot be
      // taken for an index (the values below 2^-126 stay indices, and are read
      // when they are added).
      const int32_t* more_ids = a.bias_ids + row * a.bias_stride;
      auto place = [&](int id) -> uint32_t {
        const uint32_t at = (uint32_t)id - (uint32_t)c0;
        return at < (uint32_t)kChunk && id < V ? at : ~0u;
      };
      for (int i = tid; i < n_bias; i += kThreads) {
        const uint32_t at = place(i < kThreads ? bias_id : more_ids[i]);
        if (at == ~0u) continue;
        atomicMax(&bias[at], i + 1);
      }
      __syncthreads();
      for (int i = tid; i < n_bias; i += kThreads) {
        const uint32_t at = place(i < kThreads ? bias_id : more_ids[i]);
        if (at == ~0u || bias[at] != i + 1) continue;
        const uint32_t bits = __float_as_uint(i < kThreads ? bias_value
                                                           : a.bias_values[row * a.bias_stride + i]);
        if (bits >= kBiasIndices) bias[at] = (int32_t)bits;
      }
    }
    __syncthreads();
  }
  Raw* dst = static_cast<Raw*>(a.out) + row * a.out_stride;
  float best = -INFINITY;
  int best_at = -1;
  auto step = [&](uint4& w, uint32_t allowed, int at) __attribute__((always_inline)) {
    const int v = c0 + at;
    if (v >= V) return;
    if (allowed != kAll)
      w = make_uint4(masked<F>(w.x, allowed, 0), masked<F>(w.y, allowed, 1),
                     masked<F>(w.z, allowed, 2), masked<F>(w.w, allowed, 3));
    uint32_t todo = 0;  // the touched elements
    if (count) {
      constexpr int kWords = kShort ? kPer / 2 : kPer;
      uint32_t c[kWords], any = 0;
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        c[i] = seen[(kShort ? at >> 1 : at) + i];
        any |= c[i];
      }
      if (any) {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          todo |= ((kShort ? c[i >> 1] >> (16 * (i & 1)) & 0xffffu : c[i]) != 0 ? 1u : 0u) << i;
      }
    }
    if constexpr (kBias) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) todo |= (bias[at + i] != 0 ? 1u : 0u) << i;
    }
    todo &= allowed;
    if (a.next_token) {
      // The elements that stay as they are first: among equals the lower id.
      float x[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[i] = F::up(element<F>(w, i));
      if (todo) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) x[i] = todo >> i & 1 ? -INFINITY : x[i];
      }
      float top = x[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) top = fmaxf(top, x[i]);
      if (top > best) {
        best = top;
#pragma unroll
        for (int i = kPer - 1; i >= 0; --i) best_at = x[i] == top ? v + i : best_at;
      }
    }
    while (todo) {
      const int i = __builtin_ctz(todo);
      todo &= todo - 1;
      float x = F::up(element<F>(w, i));
      uint32_t c = 0;
      if (count) {
        c = seen[kShort ? (at + i) >> 1 : at + i];
        if (kShort) c = c >> (16 * (i & 1)) & 0xffffu;
      }
      if (c) {
        x = x > 0.f ? x / rep : x * rep;
        if (c & made_bits) {
          const float f = freq * (float)(c & made_bits);
          x = x - f;
          x = x - pres;
        }
      }
      if constexpr (kBias) {
        const uint32_t b = (uint32_t)bias[at + i];
        if (b >= kBiasIndices) x = x + __uint_as_float(b);
        else if (b) x = x + a.bias_values[row * a.bias_stride + b - 1];
      }
      put<F>(w, i, F::down(x));
      if (x > best || (x == best && v + i < best_at)) {
        best = x;
        best_at = v + i;
      }
    }
  };
#pragma unroll
  for (int u = 0; u < kLoads; ++u) step(raw[u], allow[u], (u * kThreads + tid) * kPer);
  // The choice goes out before the row does: its hand-over takes two trips to
  // memory, which the stores then do not stand in front of.
  uint64_t top = 0;
  bool collects = false;
  if (choose) {
    top = wave_max(choice(best, best_at));
    if ((tid & 63) == 0) red[tid >> 6] = top;
    __syncthreads();
    collects = __builtin_amdgcn_readfirstlane(order) == (uint32_t)a.chunks - 1 && tid < 64;
    if (tid == 0) {
      for (int i = 1; i < kThreads / 64; ++i) top = max64(top, red[i]);
      if (!collects)
        __hip_atomic_store(&a.best[(int64_t)lr * a.chunks + chunk], top ? top : kNoChoice,
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int v = c0 + (u * kThreads + tid) * kPer;
    if (v < V) store_chunk<F>(dst, v, V, raw[u]);
  }
  if (!collects) return;
  top = tid == 0 ? top : 0;
  bool gave_up = false;
  for (int i = tid; i < a.chunks; i += 64) {
    if (i == chunk) continue;
    uint64_t* word = &a.best[(int64_t)lr * a.chunks + i];
    uint64_t other = 0;
    for (int spin = 0; !other; ++spin) {
      other = __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (!other && spin == kSpinLimit) {
        gave_up = true;
        break;
      }
      if (!other) __builtin_amdgcn_s_sleep(4);
    }
    __hip_atomic_store(word, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (other != kNoChoice) top = max64(top, other);
  }
  top = wave_max(top);
  const bool failed = __any(gave_up);
  if (tid == 0) {
    if (a.chunks > 1) st_u32<true>(ticket, 0);
    a.next_token[row] = failed ? -1 : chosen(top);
  }
}

// How a call is cut: threads and 16-byte loads of a workgroup.
// Four loads (a chunk of 16 KB), one where that would leave fewer than 512
// workgroups: 16 rows of 50,304 f32 logits 6.5 us with one and 8.1 with four, 64
// rows 11.3 and 10.0.  Two for 16-bit logits with biases, whose words of LDS keep
// all but three workgroups of four loads out of a CU: 90 rows of 68,149 11.0 and
// 15.7.  From kLongHistory ids on 1,024 threads count: 19 rows of 50,304 and 8,000
// ids 9.5 us and 10.6 with 256, 64 rows and 12,000 16.1 and 18.4; 132 rows of 64,066
// and 4,756 ids 26.0 and 20.2, 64 rows and 6,000 14.5 and 14.1.
struct LogitsPlan {
  int threads, loads, chunks;
};
LogitsPlan logits_plan(int32_t rows, int32_t vocab, int per, int32_t history_width, bool biases) {
  LogitsPlan p{256, biases && per == 8 ? 2 : 4, 0};
  auto chunks = [&] {
    const int64_t c = (int64_t)p.threads * per * p.loads;
    return (int)((vocab + c - 1) / c);
  };
  if (history_width >= kLongHistory) {
    p.threads = 1024;
    p.loads = 8 / per;
  } else if ((int64_t)rows * chunks() < 512) {
    p.loads = 1;
  }
  p.chunks = chunks();
  return p;
}

template <class F, int kThreads, int kLoads, int kBiasLoads = kLoads>
void launch_logits(const LogitsArg& a, unsigned blocks, hipStream_t stream) {
  if (a.bias_ids)
    hipLaunchKernelGGL((process_logits_kernel<F, kThreads, kBiasLoads, true>), dim3(blocks), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((process_logits_kernel<F, kThreads, kLoads, false>), dim3(blocks), dim3(kThreads), 0, stream, a);
}

template <class F>
void launch_type(const LogitsArg& a, const LogitsPlan& p, unsigned blocks, hipStream_t stream) {
  if (p.threads == 1024) launch_logits<F, 1024, 8 / F::kPer>(a, blocks, stream);
  else if (p.loads == 1) launch_logits<F, 256, 1>(a, blocks, stream);
  else launch_logits<F, 256, 4, F::kPer == 8 ? 2 : 4>(a, blocks, stream);
}

}  // namespace

int32_t emoe::check_process_logits(const emoe_logits_args& A, const void* workspace,
                                   size_t workspace_bytes) {
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
  if (A.history_width > (1 << 30))
    return report_error(EMOE_ESHAPE, "history_width %d above 2^30", A.history_width);
  if (A.history && many && A.history_stride < A.history_width)
    return report_error(EMOE_EINVAL, "history_stride below history_width %d", A.history_width);
  if (!A.history && (A.repetition || A.presence || A.frequency))
    return report_error(EMOE_EINVAL, "penalties without a history");
  if (!A.bias_ids != !A.bias_values)
    return report_error(EMOE_EINVAL, "one of bias_ids and bias_values is NULL");
  if (A.bias_width >= (int32_t)kBiasIndices)
    return report_error(EMOE_ESHAPE, "bias_width %d above %d", A.bias_width, (int)kBiasIndices - 1);
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
  if (A.next_token) {
    const size_t need = emoe_process_logits_workspace_bytes(A.rows, A.vocab);
    if (!workspace || workspace_bytes < need)
      return report_error(EMOE_EINVAL, "workspace of %zu bytes < %zu needed",
                          workspace ? workspace_bytes : 0, need);
    if (!aligned16(workspace)) return report_error(EMOE_EINVAL, "workspace: need 16-byte alignment");
  }
  return EMOE_OK;
}

extern "C" {

size_t emoe_process_logits_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 0 || vocab < 1) return 0;
  const size_t held = rows < kMaxRows ? rows : kMaxRows;
  return held * (kTicketLine + (((size_t)vocab + 1023) / 1024) * 8);  // the smallest chunks
}

int32_t emoe_process_logits(const emoe_logits_args* args, void* workspace, size_t workspace_bytes,
                            hipStream_t stream) {
  if (!args) return report_error(EMOE_EINVAL, "args is NULL");
  const emoe_logits_args& A = *args;
  const int32_t st = check_process_logits(A, workspace, workspace_bytes);
  if (st || A.rows == 0) return st;
  const int per = A.dtype == EMOE_F32 ? 4 : 8;
  const LogitsPlan plan = logits_plan(A.rows, A.vocab, per, A.history ? A.history_width : 0, A.bias_ids && A.bias_width > 0);
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
  a.logits_stride = A.logits_stride;
  a.out_stride = A.out_stride;
  a.history_stride = A.history_stride;
  a.bias_stride = A.bias_stride;
  a.mask_stride = A.mask_stride;
  a.vocab = A.vocab;
  a.history_width = A.history_width;
  a.bias_width = A.bias_width;
  a.n_masks = A.n_masks;
  a.chunks = plan.chunks;
  // Rows of one launch: a grid of at most 2^31 threads (plan.chunks is at most 2^18,
  // and below 2^11 with the smallest chunks: fewer than 512 of up to four times their size).
  int64_t step = ((int64_t)1 << 21) / plan.chunks;
  if (step > kMaxRows) step = kMaxRows;
  if (step > A.rows) step = A.rows;
  a.tickets = static_cast<uint32_t*>(workspace);
  a.best = reinterpret_cast<uint64_t*>(a.tickets + step * kTicketStride);
  for (int64_t r0 = 0; r0 < A.rows; r0 += step) {
    a.row0 = (int32_t)r0;
    const int64_t n = A.rows - r0 < step ? A.rows - r0 : step;
    const unsigned blocks = (unsigned)(n * plan.chunks);
    if (A.dtype == EMOE_F32) launch_type<F32>(a, plan, blocks, stream);
    else if (A.dtype == EMOE_BF16) launch_type<Half<Bf16>>(a, plan, blocks, stream);
    else launch_type<Half<Fp16>>(a, plan, blocks, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
      return report_error(EMOE_EHIP, "process_logits_kernel launch: %s", hipGetErrorString(e));
  }
  return EMOE_OK;
}

}  // extern "C"
