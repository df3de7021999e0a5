// The serving step's bookkeeping: block tables and slot maps from request lengths, and rotary positions with the new keys' and
// values' way into the cache's pages.
#include <algorithm>

#include "dyn_serve.h"

namespace {

// What a request's lengths ask for; lengths that cannot be are cut to what can, and reported.
struct Ask { int32_t ctx, n, have, need, back; bool bad, too_long; };
__device__ __forceinline__ uint32_t columns_of(const KvStepArgs& a, uint32_t tokens) { return (tokens + ((1u << a.page_shift) - 1u)) >> a.page_shift; }
__device__ __forceinline__ Ask ask_of(const KvStepArgs& a, int b) {
  Ask r;
  const int32_t c = a.ctx_len[b], n = a.new_len[b];
  const uint32_t cap = (uint32_t)a.max_pages << a.page_shift;       // below 2^31, as are both lengths: their sum is below 2^32
  r.bad = c < 0 || (uint32_t)c > cap || n < -1;
  r.ctx = (int32_t)min((uint32_t)max(c, 0), cap);
  r.have = (int32_t)columns_of(a, (uint32_t)r.ctx);
  r.back = n == -1 ? r.have : 0;
  r.n = max(n, 0);
  r.too_long = (uint32_t)r.ctx + (uint32_t)r.n > cap;
  r.need = r.too_long ? 0 : (int32_t)columns_of(a, (uint32_t)r.ctx + (uint32_t)r.n) - r.have;
  return r;
}
__device__ __forceinline__ int32_t cached_of(const KvStepArgs& a, int b) {   // -1: more tokens than the row has columns
  const Ask q = ask_of(a, b);
  return q.too_long ? -1 : q.ctx;
}

// New tokens (as an unsigned sum that stays at 2^32 - 1 once it is there: n_token is less), pages asked for, pages given back.
struct Sums { uint32_t n; int32_t need, back; };
__device__ __forceinline__ uint32_t add_sat(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }
__device__ __forceinline__ Sums operator+(const Sums& x, const Sums& y) { return {add_sat(x.n, y.n), x.need + y.need, x.back + y.back}; }

template <int CTRL, int ROWS>
__device__ __forceinline__ Sums moved(const Sums& v) {      // 0 where no lane is that far back
  return {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)v.n, CTRL, ROWS, 0xF, false), __builtin_amdgcn_update_dpp(0, v.need, CTRL, ROWS, 0xF, false),
          __builtin_amdgcn_update_dpp(0, v.back, CTRL, ROWS, 0xF, false)};
}

// Sums over the lanes up to this one; all lanes active.
__device__ __forceinline__ Sums upto_lane(Sums in) {
  in = in + moved<0x111, 0xF>(in);   // row_shr:1, 2, 4, 8: inside the rows of 16 lanes
  in = in + moved<0x112, 0xF>(in);
  in = in + moved<0x114, 0xF>(in);
  in = in + moved<0x118, 0xF>(in);
  in = in + moved<0x142, 0xA>(in);   // row_bcast:15 into rows 1 and 3
  in = in + moved<0x143, 0xC>(in);   // row_bcast:31 into rows 2 and 3
  return in;
}
__device__ __forceinline__ Sums of_lane(const Sums& v, int lane) {
  return {(uint32_t)__builtin_amdgcn_readlane((int)v.n, lane), __builtin_amdgcn_readlane(v.need, lane), __builtin_amdgcn_readlane(v.back, lane)};
}
// Sums over the waves before this one, and over all.  s_wave: one Sums per wave.
template <int WAVES>
__device__ __forceinline__ Sums before_wave(const Sums& mine, Sums* s_wave, Sums* total) {
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_wave[wave] = mine;
  __syncthreads();
  Sums base = {0, 0, 0}, all = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w == wave) base = all;
    all = all + s_wave[w];
  }
  *total = all;
  return base;
}

// The last b in [lo, hi] with at[b] <= x; at does not decrease, at[lo] <= x.
__device__ __forceinline__ int last_at(const int32_t* at, int lo, int hi, int32_t x) {
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (at[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}
// The same for an x that is the same in all lanes of a wave: 64 places at a time.
__device__ __forceinline__ int last_at_all(const int32_t* at, int lo, int hi, int32_t x) {
  const int lane = threadIdx.x & 63;
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64;
    const int k = __popcll(__ballot(at[min(lo + (lane + 1) * step, hi)] <= x));
    const int to = k == 64 ? hi : min(lo + (k + 1) * step, hi) - 1;
    lo = min(lo + k * step, hi);
    hi = max(to, lo);
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
constexpr int kStepAhead = 4;     // tokens of a thread at a time: their entries are fetched together
template <int kStepThreads>
__device__ __forceinline__ void step_items(const KvStepArgs& a, const Ring& ring, const int32_t* cu, const int32_t* need, const int32_t* back,
                                           const int32_t* s_ctx) {   // s_ctx: cached_of() of every request, or null
  const int tid = threadIdx.x, B = a.n_req, page = 1 << a.page_shift;
  const int32_t n_need = need[B], n_back = back[B], n_tok = cu[B];
  const int64_t piece = (((int64_t)a.n_token + gridDim.x - 1) / gridDim.x + kStepThreads - 1) / kStepThreads * kStepThreads;
  const int64_t p0 = blockIdx.x * piece, p1 = min(p0 + piece, (int64_t)a.n_token) - 1;
  if (p0 <= p1) {
    const int lo = last_at_all(cu, 0, B, (int32_t)p0), hi = min(last_at_all(cu, lo, B, (int32_t)p1), B - 1);
    for (int64_t t0 = p0 + tid; t0 <= p1; t0 += kStepAhead * kStepThreads) {
      int32_t pos[kStepAhead], entry[kStepAhead];
#pragma unroll
      for (int i = 0; i < kStepAhead; ++i) {
        const int64_t t = t0 + i * kStepThreads;
        pos[i] = -1;
        entry[i] = -1;
        if (t > p1 || t >= n_tok) continue;
        const int b = last_at(cu, min(lo, hi), hi, (int32_t)t);
        const int32_t c = s_ctx ? s_ctx[b] : cached_of(a, b);
        if (c < 0) continue;                         // refused: more tokens than the row has columns
        const uint32_t x = (uint32_t)c + (uint32_t)(t - cu[b]);
        const int32_t have = (int32_t)columns_of(a, (uint32_t)c), col = (int32_t)(x >> a.page_shift), want = need[b + 1] - need[b];
        if ((want && need[b + 1] > ring.count) || col >= have + want) continue;      // refused: too few pages
        entry[i] = col < have ? a.table[(size_t)b * a.max_pages + col] : a.ring[ring_at(a, ring, need[b] + col - have)];
        pos[i] = (int32_t)x;
      }
#pragma unroll
      for (int i = 0; i < kStepAhead; ++i) {
        const int64_t t = t0 + i * kStepThreads;
        if (t > p1) continue;
        a.pos[t] = pos[i];
        a.slot[t] = entry[i] >= 0 && entry[i] < a.n_page ? (entry[i] << a.page_shift) + (pos[i] & (page - 1)) : -1;
      }
    }
  }
  // this block's part of a flat range: [first, last] of the items, [lo, hi] of their requests
  auto part = [&](const int32_t* sums, int32_t count, int32_t* first, int32_t* last, int* lo, int* hi) {
    const int32_t each = (int32_t)(((int64_t)count + gridDim.x - 1) / gridDim.x);
    const int64_t from = (int64_t)blockIdx.x * each;
    if (from >= count) return false;
    *first = (int32_t)from;
    *last = (int32_t)min(from + each, (int64_t)count) - 1;
    *lo = last_at_all(sums, 0, B - 1, *first);
    *hi = last_at_all(sums, *lo, B - 1, *last);
    return true;
  };
  int32_t first, last;
  int lo, hi;
  if (part(need, n_need, &first, &last, &lo, &hi))
    for (int32_t e = first + tid; e <= last; e += kStepThreads) {
      const int b = last_at(need, lo, hi, e);
      if (need[b + 1] > ring.count) continue;
      const int32_t c = s_ctx ? s_ctx[b] : cached_of(a, b);
      const int32_t have = (int32_t)columns_of(a, (uint32_t)c);
      a.table[(size_t)b * a.max_pages + have + (e - need[b])] = a.ring[ring_at(a, ring, e)];
    }
  if (part(back, min(n_back, a.n_page - ring.count), &first, &last, &lo, &hi))
    for (int32_t e = first + tid; e <= last; e += kStepThreads) {
      const int b = last_at(back, lo, hi, e);
      a.ring[ring_at(a, ring, ring.count + e)] = a.table[(size_t)b * a.max_pages + (e - back[b])];
    }
}

// What is written once per request, and the free list's new state (by the block that has the sums).
__device__ __forceinline__ void write_request(const KvStepArgs& a, int b, const Ask& q, const Sums& before, int32_t count) {
  const bool ok = !q.too_long && (q.need == 0 || before.need + q.need <= count), gone = a.new_len[b] == -1;
  a.cu[b] = (int32_t)min(before.n, (uint32_t)a.n_token);
  a.kv_len[b] = ok && !gone ? q.ctx + q.n : 0;
  a.next_len[b] = gone ? 0 : ok ? q.ctx + q.n : q.ctx;
}
__device__ __forceinline__ uint32_t status_of(const KvStepArgs& a, const Ask& q, const Sums& before, int32_t count) {
  return (q.bad ? DYN_WS_BAD_REQUEST : 0u) | (q.too_long || (q.need && before.need + q.need > count) ? DYN_WS_NO_PAGES : 0u);
}
__device__ __forceinline__ void write_state(const KvStepArgs& a, const Ring& r, int32_t taken, const Sums& all, uint32_t status) {
  if (all.n != (uint32_t)a.n_token) status |= DYN_WS_BAD_REQUEST;
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
// few tokens is latency: the launch, the lengths, the sums, the table's entry, one after the other.  EACH: requests of a thread.
// 64 requests that generate 5.5 us, 999 mixed ones (38 000 tokens) 9.2; 3000 prompts of 1.6 million tokens together 15.9 (13 MB: 2.7 us of a copy).
template <int EACH, int kStepThreads>
__global__ __launch_bounds__(kStepThreads) void kv_step_kernel(KvStepArgs a) {
  constexpr int kMost = EACH * kStepThreads;
  __shared__ int32_t s_cu[kMost + 1], s_need[kMost + 1], s_back[kMost + 1], s_ctx[kMost];
  __shared__ Sums s_wave[kStepThreads / 64];
  __shared__ uint32_t s_status;
  __shared__ int32_t s_taken;
  const int tid = threadIdx.x, B = a.n_req;
  if (tid == 0) { s_status = 0u; s_taken = 0; }
  const Ring ring = ring_of(a);
  // a wave has EACH x 64 requests one after the other
  const int lane = tid & 63, first = (tid >> 6) * EACH * 64;
  Ask q[EACH];
  Sums at[EACH], mine = {0, 0, 0};
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int b = first + i * 64 + lane;
    q[i] = ask_of(a, min(b, B - 1));
    if (b >= B) q[i] = Ask{0, 0, 0, 0, 0, false, false};
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const Sums in = upto_lane(Sums{(uint32_t)q[i].n, q[i].need, q[i].back});
    at[i] = mine + moved<0x138, 0xF>(in);            // wave_shr:1
    mine = mine + of_lane(in, 63);
  }
  Sums all;
  const Sums base = before_wave<kStepThreads / 64>(mine, s_wave, &all);
  uint32_t status = 0;
  int32_t taken = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int b = first + i * 64 + lane;
    if (b >= B) continue;
    const Sums before = base + at[i];
    s_cu[b] = (int32_t)min(before.n, (uint32_t)a.n_token);
    s_need[b] = before.need;
    s_back[b] = before.back;
    s_ctx[b] = q[i].too_long ? -1 : q[i].ctx;
    if (blockIdx.x == 0) {
      write_request(a, b, q[i], before, ring.count);
      status |= status_of(a, q[i], before, ring.count);
      if (before.need + q[i].need <= ring.count) taken = before.need + q[i].need;
    }
  }
  if (tid == 0) {
    s_cu[B] = (int32_t)min(all.n, (uint32_t)a.n_token);
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
  step_items<kStepThreads>(a, ring, s_cu, s_need, s_back, s_ctx);
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
    const Sums in = upto_lane(Sums{(uint32_t)q.n, q.need, q.back});
    Sums all;
    const Sums at = carry + before_wave<kSumThreads / 64>(of_lane(in, 63), s_wave, &all) + moved<0x138, 0xF>(in);
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
    a.cu[B] = (int32_t)min(carry.n, (uint32_t)a.n_token);
    a.need[B] = carry.need;
    a.back[B] = carry.back;
    write_state(a, ring, s_taken, carry, s_status);
  }
}
__global__ __launch_bounds__(256) void kv_items_kernel(KvStepArgs a) {
  step_items<256>(a, ring_of(a), a.cu, a.need, a.back, nullptr);
}

}  // namespace

hipError_t dyn_launch_kv_step(const KvStepArgs& a, hipStream_t s) {
  DynTimed timed(DYN_K_KV_STEP, s);
  // a token a thread while that is at most two blocks a compute unit; requests may give back many pages each
  const int64_t pieces = std::max<int64_t>(((int64_t)a.n_token + 255) / 256, (a.n_req + 3) / 4);
  auto grid = [&](int64_t most) { return dim3((unsigned)std::min(std::max<int64_t>(pieces, 1), most)); };
  static_assert(DYN_KV_ONE_LAUNCH == 4 * 1024, "requests of a thread");
  if (a.n_req <= 256) hipLaunchKernelGGL((kv_step_kernel<1, 256>), grid(512), dim3(256), 0, s, a);
  else if (a.n_req <= 1024) hipLaunchKernelGGL((kv_step_kernel<4, 256>), grid(512), dim3(256), 0, s, a);
  else if (a.n_req <= DYN_KV_ONE_LAUNCH) hipLaunchKernelGGL((kv_step_kernel<4, 1024>), grid(512), dim3(1024), 0, s, a);
  else {
    hipLaunchKernelGGL(kv_sums_kernel, dim3(1), dim3(kSumThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kv_items_kernel, grid(2048), dim3(256), 0, s, a);
  }
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
// has 2 V elements of a head: V pairs, or 2 V elements that are not rotated.  Bound by the bytes it moves, at few tokens by latency.  4738 tokens (32 heads over
// 8, 128 wide, an 8-bit cache; 107 MB) 20.4 us, 5.2 TB/s, where a copy of 2 GiB moves 5.0; 64 tokens 4.0 us.
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
