// The serving step's bookkeeping: block tables and slot maps from request lengths, and rotary positions with the new keys' and
// values' way into the cache's pages.
#include <algorithm>

#include "dyn_serve.h"

namespace {

// What a request's lengths ask for; lengths that cannot be are cut to what can, and reported.
struct Ask { int32_t ctx, n, have, need, back; bool bad, too_long; };
__device__ __forceinline__ Ask ask_of(const KvStepArgs& a, int b) {
  Ask r;
  int32_t c = a.ctx_len[b], n = a.new_len[b];
  const int64_t cap = (int64_t)a.max_pages << a.page_shift;
  const int32_t up = (1 << a.page_shift) - 1;
  r.bad = c < 0 || c > cap || n < -1;
  c = (int32_t)min((int64_t)max(c, 0), cap);
  r.have = (int32_t)(((int64_t)c + up) >> a.page_shift);
  r.back = n == -1 ? r.have : 0;
  n = max(n, 0);
  r.too_long = (int64_t)c + n > cap;
  r.need = r.too_long ? 0 : (int32_t)(((int64_t)c + n + up) >> a.page_shift) - r.have;
  r.ctx = c;
  r.n = n;
  return r;
}

__device__ __forceinline__ int32_t cached_of(const KvStepArgs& a, int b) {   // -1: more tokens than the row has columns
  const Ask q = ask_of(a, b);
  return q.too_long ? -1 : q.ctx;
}

struct Sums { int64_t n; int32_t need, back; };
__device__ __forceinline__ Sums operator+(const Sums& x, const Sums& y) { return {x.n + y.n, x.need + y.need, x.back + y.back}; }

// Sums over the threads before this one; `total` over all.  s_wave: one Sums per wave.
template <int THREADS>
__device__ __forceinline__ Sums before_of(Sums v, Sums* s_wave, Sums* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sums in = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Sums o = {__shfl_up(in.n, d), __shfl_up(in.need, d), __shfl_up(in.back, d)};
    if (lane >= d) in = in + o;
  }
  __syncthreads();
  if (lane == 63) s_wave[wave] = in;
  __syncthreads();
  Sums base = {0, 0, 0}, all = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w == wave) base = all;
    all = all + s_wave[w];
  }
  *total = all;
  return {base.n + in.n - v.n, base.need + in.need - v.need, base.back + in.back - v.back};
}

// The last b in [lo, hi] with at[b] <= x; at does not decrease, at[lo] <= x.
__device__ __forceinline__ int last_at(const int32_t* at, int lo, int hi, int32_t x) {
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (at[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

struct Ring { int32_t first, count; };
__device__ __forceinline__ Ring ring_of(const KvStepArgs& a) {
  Ring r = {a.state[0], a.state[1]};
  if (r.first < 0 || r.first >= a.n_page) r.first = 0;
  r.count = min(max(r.count, 0), a.n_page);
  return r;
}
__device__ __forceinline__ int32_t ring_at(const KvStepArgs& a, const Ring& r, int32_t x) {   // 0 <= x < n_page
  const int64_t i = (int64_t)r.first + x;
  return (int32_t)(i >= a.n_page ? i - a.n_page : i);
}

// The new tokens' positions and slots, the new pages' entries and the released pages, each a flat range over all requests that the
// blocks take in pieces; the request of an item is found by bisection in the sums over the requests before (cu, need, back: [n_req + 1]).
// Pages handed out and pages given back lie in different parts of the ring, and what a token's slot needs of a new page is read from the
// ring, not from the table: no block waits for another.
constexpr int kStepThreads = 256, kStepPiece = 1024;
__device__ __forceinline__ void step_items(const KvStepArgs& a, const Ring& ring, const int32_t* cu, const int32_t* need, const int32_t* back,
                                           const int32_t* s_ctx) {   // s_ctx: cached_of() of every request, or null
  const int tid = threadIdx.x, B = a.n_req, page = 1 << a.page_shift;
  const int32_t n_need = need[B], n_back = back[B], n_tok = cu[B];
  for (int64_t p0 = (int64_t)blockIdx.x * kStepPiece; p0 < a.n_token; p0 += (int64_t)gridDim.x * kStepPiece) {
    const int32_t p1 = (int32_t)min(p0 + kStepPiece, (int64_t)a.n_token) - 1;
    const int lo = last_at(cu, 0, B, (int32_t)p0), hi = last_at(cu, lo, B, p1);
    for (int32_t t = (int32_t)p0 + tid; t <= p1; t += kStepThreads) {
      int32_t pos = -1, slot = -1;
      if (t < n_tok) {
        const int b = last_at(cu, lo, min(hi, B - 1), t);
        const int32_t c = s_ctx ? s_ctx[b] : cached_of(a, b);
        const int64_t x = (int64_t)c + (t - cu[b]);
        const int32_t have = (int32_t)(((int64_t)c + page - 1) >> a.page_shift), col = (int32_t)(x >> a.page_shift);
        const int32_t want = need[b + 1] - need[b];
        // refused: more tokens than the row has columns, or too few pages
        const bool ok = c >= 0 && (want == 0 || need[b + 1] <= ring.count) && col < have + want;
        if (ok) {
          const int32_t entry = col < have ? a.table[(size_t)b * a.max_pages + col] : a.ring[ring_at(a, ring, need[b] + col - have)];
          pos = (int32_t)x;
          if (entry >= 0 && entry < a.n_page) slot = (entry << a.page_shift) + (int32_t)(x & (page - 1));
        }
      }
      a.pos[t] = pos;
      a.slot[t] = slot;
    }
  }
  const int step = gridDim.x * kStepThreads, at = blockIdx.x * kStepThreads + tid;
  for (int32_t e = at; e < n_need; e += step) {
    const int b = last_at(need, 0, B - 1, e);
    if (need[b + 1] > ring.count) continue;
    const int32_t c = s_ctx ? s_ctx[b] : cached_of(a, b);
    const int32_t have = (int32_t)(((int64_t)c + page - 1) >> a.page_shift);
    a.table[(size_t)b * a.max_pages + have + (e - need[b])] = a.ring[ring_at(a, ring, e)];
  }
  for (int32_t e = at; e < min(n_back, a.n_page - ring.count); e += step) {
    const int b = last_at(back, 0, B - 1, e);
    a.ring[ring_at(a, ring, ring.count + e)] = a.table[(size_t)b * a.max_pages + (e - back[b])];
  }
}

// What is written once per request, and the free list's new state (by the block that has the sums).
__device__ __forceinline__ void write_request(const KvStepArgs& a, int b, const Ask& q, const Sums& before, int32_t count) {
  const bool ok = !q.too_long && (q.need == 0 || before.need + q.need <= count), gone = a.new_len[b] == -1;
  a.cu[b] = (int32_t)min(before.n, (int64_t)a.n_token);
  a.kv_len[b] = ok && !gone ? q.ctx + q.n : 0;
  a.next_len[b] = gone ? 0 : ok ? q.ctx + q.n : q.ctx;
}
__device__ __forceinline__ uint32_t status_of(const KvStepArgs& a, const Ask& q, const Sums& before, int32_t count) {
  return (q.bad ? DYN_WS_BAD_REQUEST : 0u) | (q.too_long || (q.need && before.need + q.need > count) ? DYN_WS_NO_PAGES : 0u);
}
__device__ __forceinline__ void write_state(const KvStepArgs& a, const Ring& r, int32_t taken, const Sums& all, uint32_t status) {
  if (all.n != a.n_token) status |= DYN_WS_BAD_REQUEST;
  if ((int64_t)r.count + all.back > a.n_page) status |= DYN_WS_BAD_PAGE;    // more pages than there are: those beyond are not taken back
  if (a.state[0] != r.first || a.state[1] != r.count) status |= DYN_WS_BAD_PAGE;
  const int64_t f = (int64_t)r.first + taken;
  a.state_out[0] = (int32_t)(f >= a.n_page ? f - a.n_page : f);
  a.state_out[1] = min(r.count + min(all.back, a.n_page - r.count), a.n_page) - taken;
  a.header->status = status;
  a.header->kind = DYN_WS_KIND_WORD;
  a.header->cells = 0;
}

// Up to DYN_KV_ONE_LAUNCH requests: every block makes all sums for itself, in LDS, and takes its pieces: one launch.  What bounds a step of
// few tokens is latency: the launch, the lengths, the sums, the table's entry, one after the other.
__global__ __launch_bounds__(kStepThreads) void kv_step_kernel(KvStepArgs a) {
  constexpr int kEach = DYN_KV_ONE_LAUNCH / kStepThreads;
  __shared__ int32_t s_cu[DYN_KV_ONE_LAUNCH + 1], s_need[DYN_KV_ONE_LAUNCH + 1], s_back[DYN_KV_ONE_LAUNCH + 1], s_ctx[DYN_KV_ONE_LAUNCH];
  __shared__ Sums s_wave[kStepThreads / 64];
  __shared__ uint32_t s_status;
  __shared__ int32_t s_taken;
  const int tid = threadIdx.x, B = a.n_req, each = (B + kStepThreads - 1) / kStepThreads;
  if (tid == 0) { s_status = 0u; s_taken = 0; }
  const Ring ring = ring_of(a);
  Ask q[kEach];
  Sums mine = {0, 0, 0};
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = tid * each + i;
    if (i < each && b < B) {
      q[i] = ask_of(a, b);
      mine = mine + Sums{q[i].n, q[i].need, q[i].back};
    }
  }
  Sums all, at = before_of<kStepThreads>(mine, s_wave, &all);
  uint32_t status = 0;
  int32_t taken = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = tid * each + i;
    if (i < each && b < B) {
      s_cu[b] = (int32_t)min(at.n, (int64_t)a.n_token);
      s_need[b] = at.need;
      s_back[b] = at.back;
      s_ctx[b] = q[i].too_long ? -1 : q[i].ctx;
      if (blockIdx.x == 0) {
        write_request(a, b, q[i], at, ring.count);
        status |= status_of(a, q[i], at, ring.count);
        if (at.need + q[i].need <= ring.count) taken = at.need + q[i].need;
      }
      at = at + Sums{q[i].n, q[i].need, q[i].back};
    }
  }
  if (tid == 0) {
    s_cu[B] = (int32_t)min(all.n, (int64_t)a.n_token);
    s_need[B] = all.need;
    s_back[B] = all.back;
  }
  if (blockIdx.x == 0) {
    if (status) atomicOr(&s_status, status);
    if (taken) atomicMax(&s_taken, taken);
  }
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) {
    a.cu[B] = s_cu[B];
    write_state(a, ring, s_taken, all, s_status);
  }
  step_items(a, ring, s_cu, s_need, s_back, s_ctx);
}

// More requests: the sums by one block, through all requests a thousand at a time, then the pieces.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void kv_sums_kernel(KvStepArgs a) {
  __shared__ Sums s_wave[kSumThreads / 64];
  __shared__ uint32_t s_status;
  __shared__ int32_t s_taken;
  const int tid = threadIdx.x, B = a.n_req;
  if (tid == 0) { s_status = 0u; s_taken = 0; }
  const Ring ring = ring_of(a);
  Sums carry = {0, 0, 0};
  uint32_t status = 0;
  int32_t taken = 0;
  for (int b0 = 0; b0 < B; b0 += kSumThreads) {
    const int b = b0 + tid;
    Ask q = {0, 0, 0, 0, 0, false, false};
    if (b < B) q = ask_of(a, b);
    Sums all;
    const Sums at = carry + before_of<kSumThreads>(Sums{q.n, q.need, q.back}, s_wave, &all);
    if (b < B) {
      write_request(a, b, q, at, ring.count);
      a.need[b] = at.need;
      a.back[b] = at.back;
      status |= status_of(a, q, at, ring.count);
      if (at.need + q.need <= ring.count) taken = at.need + q.need;
    }
    carry = carry + all;
  }
  if (status) atomicOr(&s_status, status);
  if (taken) atomicMax(&s_taken, taken);
  __syncthreads();
  if (tid == 0) {
    a.cu[B] = (int32_t)min(carry.n, (int64_t)a.n_token);
    a.need[B] = carry.need;
    a.back[B] = carry.back;
    write_state(a, ring, s_taken, carry, s_status);
  }
}
__global__ __launch_bounds__(kStepThreads) void kv_items_kernel(KvStepArgs a) {
  step_items(a, ring_of(a), a.cu, a.need, a.back, nullptr);
}

}  // namespace

hipError_t dyn_launch_kv_step(const KvStepArgs& a, hipStream_t s) {
  DynTimed timed(DYN_K_KV_STEP, s);
  const int64_t pieces = std::max<int64_t>(((int64_t)a.n_token + kStepPiece - 1) / kStepPiece, (a.n_req + 63) / 64);
  const unsigned grid = (unsigned)std::min<int64_t>(std::max<int64_t>(pieces, 1), 1024);
  if (a.n_req <= DYN_KV_ONE_LAUNCH) {
    hipLaunchKernelGGL(kv_step_kernel, dim3(grid), dim3(kStepThreads), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(kv_sums_kernel, dim3(1), dim3(kSumThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kv_items_kernel, dim3(grid), dim3(kStepThreads), 0, s, a);
  return hipGetLastError();
}

namespace {

// ---- rotary positions and the cache's new rows ---------------------------------------------------------------------

constexpr float kE4M3Max = 448.0f;

// Two values to e4m3, each rounded once to nearest even from 32 bits; beyond +-448 they are stored as +-448 (the conversion makes them NaN),
// NaN stays NaN (med3 would make it a number).
__device__ __forceinline__ uint32_t to_e4m3(float x, float y) {
  const float cx = x != x ? x : fminf(fmaxf(x, -kE4M3Max), kE4M3Max), cy = y != y ? y : fminf(fmaxf(y, -kE4M3Max), kE4M3Max);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(cx, cy, 0, false) & 0xffffu;
}

template <typename T, int V>
struct alignas(sizeof(T) * V) Pack { T x[V]; };

template <typename T, int V>
__device__ __forceinline__ void get(const T* p, float* x) {
  const Pack<T, V> r = *(const Pack<T, V>*)p;
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = (float)r.x[i];
}
template <typename T, int V>
__device__ __forceinline__ void put(T* p, const float* x) {
  Pack<T, V> r;
#pragma unroll
  for (int i = 0; i < V; ++i) r.x[i] = (T)x[i];   // rounded once, to nearest even
  *(Pack<T, V>*)p = r;
}
template <int V>
__device__ __forceinline__ void put8(uint8_t* p, const float* x, float scale) {
  if constexpr (V == 1) {
    *p = (uint8_t)to_e4m3(x[0] / scale, 0.0f);
  } else {
    uint32_t w[(V + 3) / 4] = {};
#pragma unroll
    for (int i = 0; i < V; i += 2) w[i / 4] |= to_e4m3(x[i] / scale, x[i + 1] / scale) << (8 * (i % 4));
    Pack<uint32_t, (V + 3) / 4> r;
#pragma unroll
    for (int i = 0; i < (V + 3) / 4; ++i) r.x[i] = w[i];
    *(Pack<uint32_t, (V + 3) / 4>*)p = r;
  }
}

// (x_i, x_j) -> (x_i c - x_j s, x_j c + x_i s) for the pairs of the first `rotary` elements of every query and key head, the rest as it is; keys
// and values into the slot's row of the cache.  A block has one token and a part of its heads; the token's angles once, in LDS: position x turns
// per position in 64 bits, of which only the fraction of a turn counts (exact to 2^-22 of a turn at position 2^31), sine and cosine in 32.  A thread
// has 2 V elements of a head: V pairs, or 2 V elements that are not rotated.  Bound by the bytes it moves, at few tokens by latency.
template <typename T, bool F8, int V>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeArgs a) {
  __shared__ float s_cos[DYN_ROPE_MAX_PAIRS], s_sin[DYN_ROPE_MAX_PAIRS];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, D = a.head_dim, pairs = a.rotary / 2;
  const int32_t pos = a.pos[t], slot = a.slot[t];
  if (tid < pairs) {
    const double turns = (double)pos * a.turn[tid];
    const float f = (float)(turns - rint(turns));
    float c, s;
    sincospif(2.0f * f, &s, &c);
    s_cos[tid] = c * a.amplitude;
    s_sin[tid] = s * a.amplitude;
  }
  __syncthreads();
  const int per = D / (2 * V), rot = pairs / V;       // units of a head, units that are rotated
  const int heads = a.n_q_head + 2 * a.n_kv_head;
  const bool stored = slot >= 0 && slot < a.n_slot;
  for (int u = blockIdx.y * 256 + tid; u < heads * per; u += gridDim.y * 256) {
    const int head = u / per, i = u % per;
    const int h = head < a.n_q_head ? head : head < a.n_q_head + a.n_kv_head ? head - a.n_q_head : head - a.n_q_head - a.n_kv_head;
    const bool is_q = head < a.n_q_head, is_v = head >= a.n_q_head + a.n_kv_head;
    const T* src = is_q ? (const T*)a.q + t * a.q_token + h * a.q_head
                 : is_v ? (const T*)a.v + t * a.v_token + h * a.v_head : (const T*)a.k + t * a.k_token + h * a.k_head;
    const bool turned = !is_v && i < rot;
    // the unit's two runs of V elements: for pairs half the rotated part apart, otherwise one after the other
    const int d0 = turned && !a.interleaved ? i * V : i * 2 * V, d1 = turned && !a.interleaved ? d0 + pairs : d0 + V;
    float x[2 * V];
    get<T, V>(src + d0, x);
    get<T, V>(src + d1, x + V);
    if (turned) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float c = s_cos[i * V + j], s = s_sin[i * V + j];
        float& lo = a.interleaved ? x[2 * j] : x[j];
        float& hi = a.interleaved ? x[2 * j + 1] : x[V + j];
        const float p = lo, q = hi;
        lo = __builtin_fmaf(p, c, -(q * s));
        hi = __builtin_fmaf(q, c, p * s);
      }
    }
    if (is_q) {
      T* dst = (T*)a.q_out + t * a.o_token + h * a.o_head;
      put<T, V>(dst + d0, x);
      put<T, V>(dst + d1, x + V);
    } else if (stored) {
      const int64_t row = ((((int64_t)(slot >> a.page_shift) * a.n_kv_head + h) << a.page_shift) + (slot & ((1 << a.page_shift) - 1))) * D;
      if constexpr (F8) {
        uint8_t* dst = (uint8_t*)(is_v ? a.v_cache : a.k_cache) + row;
        const float* scales = is_v ? a.v_scale : a.k_scale;
        const float scale = scales ? scales[h] : 1.0f;
        put8<V>(dst + d0, x, scale);
        put8<V>(dst + d1, x + V, scale);
      } else {
        T* dst = (T*)(is_v ? a.v_cache : a.k_cache) + row;
        put<T, V>(dst + d0, x);
        put<T, V>(dst + d1, x + V);
      }
    }
  }
}

template <typename T, bool F8>
hipError_t launch_rope(const RopeArgs& a, hipStream_t s) {
  const int units = (a.n_q_head + 2 * a.n_kv_head) * (a.head_dim / (2 * a.vec));
  const int parts = std::min((units + 255) / 256, std::max(1, 1024 / a.n_token));
  const dim3 grid((unsigned)a.n_token, (unsigned)parts);
  if (a.vec == 8) hipLaunchKernelGGL((rope_append_kernel<T, F8, 8>), grid, dim3(256), 0, s, a);
  else if (a.vec == 4) hipLaunchKernelGGL((rope_append_kernel<T, F8, 4>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((rope_append_kernel<T, F8, 1>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t dyn_launch_rope_append(const RopeArgs& a, hipStream_t s) {
  DynTimed timed(DYN_K_ROPE_APPEND, s);
  const bool f8 = a.cache_type == DYN_T_E4M3;
  if (a.type == DYN_T_BF16) return f8 ? launch_rope<__bf16, true>(a, s) : launch_rope<__bf16, false>(a, s);
  return f8 ? launch_rope<_Float16, true>(a, s) : launch_rope<_Float16, false>(a, s);
}
