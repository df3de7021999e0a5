// Attention of each request's new tokens over its pages of the key/value cache.
//
// Row (token i of request b, query head h) stands at p = kv_len - n + i and sees the keys j <= p with j > p - window or j < n_sink:
//   o = sum_j exp(c q.k_j - m) v_j / sum_j exp(c q.k_j - m),   c = scale x the key head's scale,
// in one pass over the keys in tiles, with a running reference m, sum and weighted sum per row, all in 32 bits.
//
// The rows of the query heads that share a key head are taken together (new tokens x group rows a key head), so that a tile of keys is read once
// for all of them.  A wave has 32 rows.  S^T = K Q^T by 32x32x16 matrix instructions: a lane then holds keys of ONE row (column lane % 32), the
// row's maximum and sum need one exchange with the lane 32 away, and, with the keys of a tile put into the instruction's rows with bits 2 and 3 of
// their index swapped, the sixteen-bit weights stand where the second product O^T = V^T P^T takes its right operand: no weight moves between lanes.
// V^T is read from LDS by the transposing read (4 keys x 16 elements for 16 lanes).  The weights are rounded to the queries' type for that product
// (the output is rounded to it too; their sum is taken before that, in 32 bits).
//
// The reference m is not the maximum itself: it is raised only when a row's maximum passes it by 2^8 in the weights, since raising it costs a
// multiplication of the whole weighted sum; weights up to 2^8 (in fp16 2^15, with 2^7 for the reference itself, so that small weights stay above
// what fp16 can hold) round as well as those up to 1.
//
// Keys that a row does not see get weight 0 by selection, whatever their score is.  A weight of 0 does not keep a value that is infinite or not a
// number out of the matrix product, so in tiles in which a row does not see every key such values are taken out on the way to LDS and given to the
// rows that see them one by one.
#include <algorithm>

#include "dyn_serve.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
using x8 = T __attribute__((ext_vector_type(8)));
template <typename T>
using x4 = T __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mfma(x8<__bf16> a, x8<__bf16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma(x8<_Float16> a, x8<_Float16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

template <typename T> struct Kind;
template <> struct Kind<__bf16> {
  static constexpr float bias = 0.0f;                     // log2 of the reference's own weight
  static constexpr uint32_t carry = 0x00800080u;          // added to the bits without sign, bit 15 tells an exponent of all ones
  static constexpr uint32_t fraction = 0x007f007fu;
  static constexpr uint32_t one = 0x3f80u;
};
template <> struct Kind<_Float16> {
  static constexpr float bias = 7.0f;
  static constexpr uint32_t carry = 0x04000400u;
  static constexpr uint32_t fraction = 0x03ff03ffu;
  static constexpr uint32_t one = 0x3c00u;
};
constexpr float kRaise = 8.0f;

// 16 bytes of a row, as they lie in the cache: 8 elements of 16 bits, or 16 of 8.  What LDS holds is 16 bits either way (every e4m3 value is one of
// both types).
__device__ __forceinline__ u32x4 widen(__bf16, uint32_t lo, uint32_t hi) {
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  const v2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const v2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
}
__device__ __forceinline__ u32x4 widen(_Float16, uint32_t lo, uint32_t hi) {
  typedef _Float16 v2 __attribute__((ext_vector_type(2)));
  const v2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
  const v2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  return u32x4{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
}

// Where 8 elements (16 bytes) of a tile lie in LDS, in units of 16 bytes: rows one after the other, the position in the row turned by the row so that the
// 16 lanes of a read hit all 64 banks: 16 keys' same elements of K, 4 keys' 32 neighbouring elements of V.
template <int DP>
__device__ __forceinline__ int k_at(int key, int c8) {
  return DP == 128 ? key * 16 + (c8 ^ (key & 15)) : key * 8 + (c8 ^ ((key >> 1) & 7));
}
template <int DP>
__device__ __forceinline__ int v_at(int key, int c8) {
  return DP == 128 ? key * 16 + (c8 ^ ((key & 3) << 2)) : key * 8 + (c8 ^ (((key >> 1) & 1) << 2));
}

// What the waves of a block share of a request: the keys its row tile sees, as tiles of KT keys without those between the first tokens and the window.
struct Keys {
  int32_t sink_tiles, first;  // tile v is v below sink_tiles, else v - sink_tiles + first
  int32_t count;
};
template <int KT>
__device__ __forceinline__ Keys keys_of(const AttnArgs& a, int32_t lo, int32_t hi) {   // positions of the first and last row, hi >= 0
  Keys k = {0, 0, hi / KT + 1};
  if (a.window > 0) {
    const int32_t first = max(0, lo - a.window + 1) / KT, sinks = (int32_t)(((int64_t)a.n_sink + KT - 1) / KT);
    if (first > sinks) {
      k.sink_tiles = sinks;
      k.first = first;
      k.count = sinks + hi / KT - first + 1;
    }
  }
  return k;
}
__device__ __forceinline__ int32_t tile_of(const Keys& k, int32_t v) { return v < k.sink_tiles ? v : v - k.sink_tiles + k.first; }

// Whether some row from position `first` to `last` does not see every key of a tile.
template <int KT>
__device__ __forceinline__ bool hides(const AttnArgs& a, int32_t first, int32_t last, int32_t key0) {
  return key0 + KT - 1 > first || (a.window > 0 && key0 <= last - a.window && key0 + KT > a.n_sink);
}

// One wave's 32 rows and what it has summed up for them.
template <typename T, int DP>
struct Rows {
  x8<T> q[DP / 16];           // right operand of the first product
  f32x16 o[DP / 32];          // O^T: column lane % 32, element 32 t + 8 (i / 4) + 4 (lane / 32) + i % 4
  float m, sum, c;            // reference (before c), sum of this lane's weights, log2(e) x scale x key scale
  int32_t pos, low;           // position (-1: no row), last key that the window hides
  int32_t first, last;        // least and greatest position in the wave
};

// One tile of KT keys from LDS (16-bit, laid out by k_at and v_at).  `key0`: the first key's position; `marks`: two bits of every value (Stage::write), or null.
template <typename T, int DP, int KT>
__device__ __forceinline__ void take_tile(const AttnArgs& a, Rows<T, DP>& r, const u32x4* lds_k, const u32x4* lds_v, const uint32_t* marks, int32_t key0) {
  const int lane = threadIdx.x & 63, n32 = lane & 31, h = lane >> 5;
  if (key0 > r.last) return;
  const bool some_hidden = hides<KT>(a, r.first, r.last, key0);
  // the keys of this lane's row that the window hides end at r.low
  if (a.window > 0 && key0 + KT - 1 <= r.first - a.window && key0 >= a.n_sink) return;
  f32x16 s[KT / 32];
#pragma unroll
  for (int mt = 0; mt < KT / 32; ++mt) {
    const int key = 32 * mt + ((n32 & 0x13) | ((n32 & 4) << 1) | ((n32 & 8) >> 1));   // bits 2 and 3 swapped
    f32x16 acc = {};
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) acc = mfma(__builtin_bit_cast(x8<T>, lds_k[k_at<DP>(key, 2 * d + h)]), r.q[d], acc);
    s[mt] = acc;
  }
  // register i of s[mt] is key 32 mt + 16 (i / 8) + 8 h + i % 8.  What a row does not see scores -inf: weight 0 below, whatever the reference.
  if (some_hidden) {
    const int32_t from = r.low - key0 - 8 * h, sinks = a.n_sink - key0 - 8 * h, upto = r.pos - key0 - 8 * h;
    if (a.window > 0) {
#pragma unroll
      for (int mt = 0; mt < KT / 32; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int32_t at = 32 * mt + 16 * (i / 8) + i % 8;
          s[mt][i] = at > upto || (at <= from && at >= sinks) ? -INFINITY : s[mt][i];
        }
    } else {
#pragma unroll
      for (int mt = 0; mt < KT / 32; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[mt][i] = 32 * mt + 16 * (i / 8) + i % 8 > upto ? -INFINITY : s[mt][i];
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int mt = 0; mt < KT / 32; ++mt)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[mt][i]);
  top = fmaxf(top, __shfl_xor(top, 32));
  const bool raise = (top - r.m) * r.c > kRaise || (r.m == -INFINITY && top > -INFINITY);
  if (__any(raise)) {
    const float m = fmaxf(r.m, top);
    const float f = r.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((r.m - m) * r.c);
    r.m = m;
    r.sum *= f;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) r.o[t][i] *= f;
  }
  const float base = Kind<T>::bias - (r.m == -INFINITY ? 0.0f : r.m * r.c);
  x8<T> p[KT / 16];
  float sum = 0.0f;
#pragma unroll
  for (int mt = 0; mt < KT / 32; ++mt)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][i], r.c, base));
      sum += w;
      p[2 * mt + i / 8][i % 8] = (T)w;
    }
  r.sum += sum;

  // V^T: lane group lane / 16 has elements 16 (group % 2) + .. of keys 8 (group / 2) + ..; two reads of 4 keys make the 8 of a lane
  const int g16 = lane >> 4, i16 = lane & 15;
  auto value = [&](int st, int t) {
    const int key = 16 * st + 8 * (g16 >> 1) + (i16 >> 2), c8 = 4 * t + 2 * (g16 & 1) + ((i16 & 3) >> 1);
    typedef __attribute__((address_space(3))) s16x4* lds4;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)((const s16x4*)&lds_v[v_at<DP>(key, c8)] + (i16 & 1)));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)((const s16x4*)&lds_v[v_at<DP>(key + 4, c8)] + (i16 & 1)));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
#pragma unroll
  for (int st = 0; st < KT / 16; ++st)
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) r.o[t] = mfma(__builtin_bit_cast(x8<T>, value(st, t)), p[st], r.o[t]);
  // Values of this tile that are not finite were taken out of it and marked: they go to the rows that see their keys.
  if (marks) {
    uint32_t any = 0;
    for (int i = lane; i < 2 * KT * DP / 32; i += 64) any |= marks[i];
    if (__any(any != 0)) {
      for (int key = 0; key < KT; ++key) {
        const int32_t at = key0 + key;
        const bool sees = at <= r.pos && (at > r.low || at < a.n_sink);
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) {
          const uint32_t up = marks[key * (DP / 32) + t] >> 4 * h, down = marks[(KT + key) * (DP / 32) + t] >> 4 * h;
          if (!__any(up | down)) continue;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int bit = 8 * (i / 4) + i % 4;
            const float x = (up >> bit & 1u ? INFINITY : 0.0f) - (down >> bit & 1u ? INFINITY : 0.0f);   // both: not a number
            r.o[t][i] += sees ? x : 0.0f;
          }
        }
      }
    }
  }
}

// A request as a block sees it; lengths and offsets are cut to what the arrays hold.
struct Request { int32_t t0, n, len; };
__device__ __forceinline__ Request request_of(const AttnArgs& a, int b) {
  Request q;
  q.t0 = min(max(a.cu[b], 0), a.n_token);
  q.n = max(min(a.cu[b + 1], a.n_token) - q.t0, 0);
  q.len = (int32_t)min((int64_t)max(a.kv_len[b], 0), (int64_t)a.max_pages << a.page_shift);
  return q;
}

// Loads one wave's rows: rows base .. base + 31 of the request's `rows` for key head kvh.
template <typename T, int DP>
__device__ __forceinline__ void load_rows(const AttnArgs& a, const Request& q, int kvh, int32_t base, int32_t rows, Rows<T, DP>& r) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int32_t row = base + (lane & 31);
  const bool in = row < rows;
  const int32_t i = (in ? row : base) / a.group, g = (in ? row : base) - i * a.group;
  const float ks = a.k_scale ? a.k_scale[kvh] : 1.0f;
  float c = a.scale * ks * 1.4426950408889634f;
  const T* src = (const T*)a.q + (int64_t)(q.t0 + i) * a.q_token + (int64_t)(kvh * a.group + g) * a.q_head;
  const uint32_t flip = c < 0.0f ? 0x80008000u : 0u;   // the reference is a maximum: a negative factor goes into the queries, exactly
  r.c = fmaxf(fabsf(c), 1e-30f);                        // above 0: -inf times it is -inf
#pragma unroll
  for (int d = 0; d < DP / 16; ++d) {
    u32x4 v = {0u, 0u, 0u, 0u};
    const int at = 16 * d + 8 * h;
    if (in && 16 * d < a.head_dim) {
      if (a.q_vec) {
        v = *(const u32x4*)(src + at);
      } else {
        const uint16_t* p = (const uint16_t*)(src + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = p[2 * j] | (uint32_t)p[2 * j + 1] << 16;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] ^= flip;
    }
    r.q[d] = __builtin_bit_cast(x8<T>, v);
  }
  r.pos = in ? q.len - q.n + i : -1;
  r.low = a.window > 0 ? r.pos - a.window : -1;
  r.first = q.len - q.n + base / a.group;
  r.last = q.len - q.n + (min(base + 31, rows - 1)) / a.group;
  r.m = -INFINITY;
  r.sum = 0.0f;
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) r.o[t] = f32x16{};
}

// 4 neighbouring elements of an output row.
template <typename T>
__device__ __forceinline__ void store4(T* p, const float* x, bool vec) {
  if (vec) {
    x4<T> v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (T)x[i];
    *(x4<T>*)p = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = (T)x[i];
  }
}

// Where a row's pieces lie: token and head.
__device__ __forceinline__ int64_t part_row(const AttnArgs& a, int chunk, int64_t t, int head) {
  return ((int64_t)chunk * a.n_token + t) * (a.n_kv_head * a.group) + head;
}

// The block that is the last of a row tile's `pieces` joins them.  Every block's pieces are written before its arrival counts (the fence), and
// the last one leaves the count as it found it, 0.  The order of the sum is that of the pieces: the same values on every run.
__device__ __forceinline__ bool last_of(uint32_t* arrived, uint32_t pieces, uint32_t* s_flag) {
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t before = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    *s_flag = before + 1u == pieces;
    if (before + 1u == pieces) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!*s_flag) return false;
  __threadfence();
  return true;
}
template <typename T>
__device__ __forceinline__ void join_rows(const AttnArgs& a, const Request& q, int kvh, int32_t base, int32_t n_row, int pieces) {
  const int quads = a.head_dim / 4;
  const float ks = a.k_scale ? a.k_scale[kvh] : 1.0f, vs = a.v_scale ? a.v_scale[kvh] : 1.0f;
  const float c = fmaxf(fabsf(a.scale * ks * 1.4426950408889634f), 1e-30f);
  for (int u = threadIdx.x; u < n_row * quads; u += blockDim.x) {
    const int32_t row = base + u / quads, i = row / a.group, d = (u % quads) * 4;
    const int head = kvh * a.group + (row - i * a.group);
    const int64_t t = q.t0 + i;
    float m = -INFINITY;
    for (int p = 0; p < pieces; ++p) m = fmaxf(m, a.part_ml[2 * part_row(a, p, t, head)]);
    float sum = 0.0f, x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p = 0; p < pieces; ++p) {
      const int64_t at = part_row(a, p, t, head);
      const float mp = a.part_ml[2 * at], f = mp == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mp - m) * c);
      sum = __builtin_fmaf(a.part_ml[2 * at + 1], f, sum);
      const float4 v = *(const float4*)(a.part + at * a.head_dim + d);
      // a piece without a weight has no part: its factor may not meet a value that is not finite
      if (mp == -INFINITY) continue;
      x[0] = __builtin_fmaf(v.x, f, x[0]);
      x[1] = __builtin_fmaf(v.y, f, x[1]);
      x[2] = __builtin_fmaf(v.z, f, x[2]);
      x[3] = __builtin_fmaf(v.w, f, x[3]);
    }
    const bool none = q.len - q.n + i < 0;
    const float by = vs / sum;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = none ? 0.0f : x[j] * by;
    store4<T>((T*)a.out + t * a.o_token + (int64_t)head * a.o_head + d, x, a.o_vec);
  }
}

// The rows' pages: an entry outside the cache is read as page 0 and reported.
__device__ __forceinline__ int32_t page_of(const AttnArgs& a, int b, int32_t key) {
  const int32_t e = a.table[(size_t)b * a.max_pages + (key >> a.page_shift)];
  if ((uint32_t)e >= (uint32_t)a.n_page) {
    atomicOr(&a.header->status, DYN_WS_BAD_PAGE);
    return 0;
  }
  return e;
}

// The part of a tile that one lane of `LANES` carries from the cache to LDS.
template <typename T, bool F8, int DP, int KT, int LANES>
struct Stage {
  static constexpr int kPerRow = F8 ? DP / 16 : DP / 8;        // 16-byte pieces of a row
  static constexpr int kEach = KT * kPerRow / LANES;           // pieces of a lane
  static_assert(KT * kPerRow % LANES == 0 && LANES % kPerRow == 0, "pieces");
  u32x4 k[kEach], v[kEach];
  // `page`: lane l of the wave has the page of key l of the tile.  Keys beyond the request's last one are read as the last one (no row sees them),
  // pieces beyond the head's end as its first piece, and K's as zeros then.
  __device__ __forceinline__ void load(const AttnArgs& a, int kvh, int32_t key0, int32_t len, int32_t page, int at) {
    const int row_bytes = a.head_dim * (F8 ? 1 : 2);
    const int c = at % kPerRow;
    const bool in = c * 16 < row_bytes;
    const int64_t head = (int64_t)kvh << a.page_shift, per_page = (int64_t)a.n_kv_head << a.page_shift;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int row = at / kPerRow + i * (LANES / kPerRow);
      const int32_t key = min(key0 + row, len - 1);
      const int64_t off = (__shfl(page, row) * per_page + head + (key & ((1 << a.page_shift) - 1))) * row_bytes + (in ? c * 16 : 0);
      k[i] = *(const u32x4*)((const char*)a.k_cache + off);
      v[i] = *(const u32x4*)((const char*)a.v_cache + off);
    }
    if (row_bytes < 16 * kPerRow) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) k[i] = in ? k[i] : u32x4{0u, 0u, 0u, 0u};
    }
  }
  // With `marks`, the values that are not finite are written as 0 and marked, a bit for +inf (the first KT rows of DP bits) and one for -inf (the others), both
  // for what is not a number: see take_tile.
  __device__ __forceinline__ void write(u32x4* lds_k, u32x4* lds_v, uint8_t* marks, int at) {
    const int c = at % kPerRow;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int row = at / kPerRow + i * (LANES / kPerRow);
      if constexpr (F8) {
        lds_k[k_at<DP>(row, 2 * c)] = widen(T{}, k[i][0], k[i][1]);
        lds_k[k_at<DP>(row, 2 * c + 1)] = widen(T{}, k[i][2], k[i][3]);
        put_v(lds_v, marks, row, 2 * c, widen(T{}, v[i][0], v[i][1]));
        put_v(lds_v, marks, row, 2 * c + 1, widen(T{}, v[i][2], v[i][3]));
      } else {
        lds_k[k_at<DP>(row, c)] = k[i];
        put_v(lds_v, marks, row, c, v[i]);
      }
    }
  }
  static __device__ __forceinline__ void put_v(u32x4* lds_v, uint8_t* marks, int row, int c8, u32x4 x) {
    if (marks) {
      uint32_t up = 0, down = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t bits = x[i], odd = (((bits & 0x7fff7fffu) + Kind<T>::carry) & 0x80008000u) >> 15;           // 1 in the halves that are not finite
        const uint32_t nan = (((bits & Kind<T>::fraction) + 0x7fff7fffu) & 0x80008000u) >> 15, neg = (bits >> 15) & 0x00010001u;
        const uint32_t u = odd & (nan | (neg ^ 0x00010001u)), d = odd & (nan | neg);
        up |= ((u | u >> 15) & 3u) << 2 * i;
        down |= ((d | d >> 15) & 3u) << 2 * i;
        x[i] = bits & ~(odd * 0xffffu);
      }
      marks[row * (DP / 8) + c8] = (uint8_t)up;
      marks[(KT + row) * (DP / 8) + c8] = (uint8_t)down;
    }
    lds_v[v_at<DP>(row, c8)] = x;
  }
};

// Requests of at most 32 rows a key head (one new token, or a few): four waves take the tiles of a piece of the keys in turn, each for all rows, and
// join at the end.  Bound by the bytes of K and V.
template <typename T, bool F8, int DP>
__global__ __launch_bounds__(256, 2) void attend_narrow_kernel(AttnArgs a) {
  constexpr int KT = DYN_ATTN_KEYS_NARROW, kTile = KT * DP / 8;     // 16-byte pieces of K (or V) of a tile
  __shared__ u32x4 s_tile[4][2 * kTile];
  __shared__ uint32_t s_marks[4][2 * KT * DP / 32];
  __shared__ float s_m[4][32], s_sum[4][32];
  __shared__ uint32_t s_flag;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.n_kv_head, b = blockIdx.x / a.n_kv_head, chunk = blockIdx.y;
  if (blockIdx.x == 0 && chunk == 0 && tid == 0) a.header->kind = DYN_WS_KIND_WORD;
  const Request q = request_of(a, b);
  const int64_t all_rows = (int64_t)q.n * a.group;
  if (q.n == 0 || all_rows > DYN_ATTN_ROWS) return;
  const int32_t rows = (int32_t)all_rows, hi = q.len - 1;
  const Keys keys = hi >= 0 ? keys_of<KT>(a, q.len - q.n, hi) : Keys{0, 0, 0};
  const int pieces = max(1, min(a.n_chunk_narrow, (keys.count + a.tiles_narrow - 1) / a.tiles_narrow));
  if (chunk >= pieces) return;
  const int32_t v0 = chunk * a.tiles_narrow, v1 = chunk == a.n_chunk_narrow - 1 ? keys.count : min(keys.count, v0 + a.tiles_narrow);
  Rows<T, DP> r;
  load_rows<T, DP>(a, q, kvh, 0, rows, r);
  u32x4* lds_k = s_tile[wave];
  u32x4* lds_v = s_tile[wave] + kTile;
  Stage<T, F8, DP, KT, 64> st;
  auto page_at = [&](int32_t v) {
    const int32_t key = min(tile_of(keys, v) * KT + (lane & (KT - 1)), q.len - 1);
    return page_of(a, b, key);
  };
  int32_t v = v0 + wave;
  if (v < v1) {
    st.load(a, kvh, tile_of(keys, v) * KT, q.len, page_at(v), lane);
    int32_t page = v + 4 < v1 ? page_at(v + 4) : 0;
    for (; v < v1; v += 4) {
      const int32_t key0 = tile_of(keys, v) * KT;
      uint32_t* marks = hides<KT>(a, r.first, r.last, key0) ? s_marks[wave] : nullptr;
      st.write(lds_k, lds_v, (uint8_t*)marks, lane);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (v + 4 < v1) {
        st.load(a, kvh, tile_of(keys, v + 4) * KT, q.len, page, lane);
        if (v + 8 < v1) page = page_at(v + 8);
      }
      take_tile<T, DP, KT>(a, r, lds_k, lds_v, marks, key0);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
  // the four waves' sums: O of each in its own tile's place, row by row
  float* s_o = (float*)s_tile[wave];
  const int row = lane & 31, h = lane >> 5;
  const float sum = r.sum + __shfl_xor(r.sum, 32);
  if (h == 0) { s_m[wave][row] = r.m; s_sum[wave][row] = sum; }
  if (row < rows) {
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(float4*)&s_o[row * DP + 32 * t + 8 * (i / 4) + 4 * h] = float4{r.o[t][i], r.o[t][i + 1], r.o[t][i + 2], r.o[t][i + 3]};
  }
  __syncthreads();
  const int quads = a.head_dim / 4;
  const float vs = a.v_scale ? a.v_scale[kvh] : 1.0f;
  for (int u = tid; u < rows * quads; u += 256) {
    const int rw = u / quads, d = (u % quads) * 4, i = rw / a.group, head = kvh * a.group + (rw - i * a.group);
    const int64_t t = q.t0 + i;
    const float m = fmaxf(fmaxf(s_m[0][rw], s_m[1][rw]), fmaxf(s_m[2][rw], s_m[3][rw]));
    float total = 0.0f, x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mw = s_m[w][rw];
      if (mw == -INFINITY && s_sum[w][rw] == 0.0f) continue;        // no weight in this wave's tiles
      const float f = mw == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((mw - m) * r.c);
      total = __builtin_fmaf(s_sum[w][rw], f, total);
      const float4 o = *(const float4*)&((const float*)s_tile[w])[rw * DP + d];
      x[0] = __builtin_fmaf(o.x, f, x[0]);
      x[1] = __builtin_fmaf(o.y, f, x[1]);
      x[2] = __builtin_fmaf(o.z, f, x[2]);
      x[3] = __builtin_fmaf(o.w, f, x[3]);
    }
    if (pieces == 1) {
      const bool none = q.len - q.n + i < 0;
      const float by = vs / total;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = none ? 0.0f : x[j] * by;
      store4<T>((T*)a.out + t * a.o_token + (int64_t)head * a.o_head + d, x, a.o_vec);
    } else {
      const int64_t at = part_row(a, chunk, t, head);
      *(float4*)(a.part + at * a.head_dim + d) = float4{x[0], x[1], x[2], x[3]};
      if (d == 0) { a.part_ml[2 * at] = m; a.part_ml[2 * at + 1] = total; }
    }
  }
  if (pieces > 1 && last_of(a.arrived_narrow + blockIdx.x, (uint32_t)pieces, &s_flag)) join_rows<T>(a, q, kvh, 0, rows, pieces);
}

// Requests of more rows: a block has 32 rows for each of its waves, all waves read the same tiles of 64 keys from LDS, two tiles in turn, the next
// one's loads in flight while one is worked on.  Bound by the matrix instructions and the exponentials beside them.
template <typename T, bool F8, int DP>
__global__ __launch_bounds__(64 * DYN_ATTN_WAVES_WIDE, 2) void attend_wide_kernel(AttnArgs a) {
  constexpr int KT = DYN_ATTN_KEYS_WIDE, NW = DYN_ATTN_WAVES_WIDE, R = 32 * NW, kTile = KT * DP / 8;
  __shared__ u32x4 s_tile[2][2 * kTile];
  __shared__ uint32_t s_marks[2][2 * KT * DP / 32];
  __shared__ uint32_t s_flag;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.n_kv_head, chunk = blockIdx.y;
  if (blockIdx.x == 0 && chunk == 0 && tid == 0) a.header->kind = DYN_WS_KIND_WORD;
  // row tiles are numbered so that request b's begin at cu[b] x group / R + b: the request of a tile follows from cu alone.  Later tiles have more
  // keys: they come first.
  const int32_t tile = a.n_tile_wide - 1 - blockIdx.x / a.n_kv_head;
  int lo = 0, hi_b = a.n_req - 1;
  auto begin_of = [&](int b) { return (int64_t)min(max(a.cu[b], 0), a.n_token) * a.group / R + b; };
  while (lo < hi_b) {   // 64 places at a time
    const int span = hi_b - lo, step = (span + 63) / 64, at = min(lo + (lane + 1) * step, hi_b);
    const unsigned long long below = __ballot(begin_of(at) <= tile);
    const int k = __popcll(below);      // the places are in order: the first k are at or before the tile
    const int nlo = k == 0 ? lo : min(lo + k * step, hi_b), nhi = k == 64 ? hi_b : min(min(lo + (k + 1) * step, hi_b) - 1, hi_b);
    lo = nlo;
    hi_b = max(nhi, nlo);
  }
  const int b = lo;
  const Request q = request_of(a, b);
  const int64_t all_rows = (int64_t)q.n * a.group, base64 = ((int64_t)tile - begin_of(b)) * R;
  if (all_rows <= DYN_ATTN_ROWS || base64 < 0 || base64 >= all_rows) return;
  const int32_t rows = (int32_t)all_rows, base = (int32_t)base64, n_row = min(R, rows - base);
  const int32_t first = q.len - q.n + base / a.group, last = q.len - q.n + (base + n_row - 1) / a.group;
  const Keys keys = last >= 0 ? keys_of<KT>(a, first, last) : Keys{0, 0, 0};
  const int pieces = max(1, min(a.n_chunk_wide, (keys.count + a.tiles_wide - 1) / a.tiles_wide));
  if (chunk >= pieces) return;
  const int32_t v0 = chunk * a.tiles_wide, v1 = chunk == a.n_chunk_wide - 1 ? keys.count : min(keys.count, v0 + a.tiles_wide);
  Rows<T, DP> r;
  const bool idle = base + 32 * wave >= rows;
  load_rows<T, DP>(a, q, kvh, idle ? 0 : base + 32 * wave, idle ? 0 : rows, r);
  if (idle) r.last = -1;
  Stage<T, F8, DP, KT, 64 * NW> st;
  auto page_at = [&](int32_t v) {
    const int32_t key = min(tile_of(keys, v) * KT + lane, q.len - 1);
    return page_of(a, b, key);
  };
  if (v0 < v1) {
    st.load(a, kvh, tile_of(keys, v0) * KT, q.len, page_at(v0), tid);
    int32_t page = v0 + 1 < v1 ? page_at(v0 + 1) : 0;
    auto marks_of = [&](int32_t v) { return hides<KT>(a, first, last, tile_of(keys, v) * KT) ? s_marks[(v - v0) & 1] : nullptr; };
    st.write(s_tile[0], s_tile[0] + kTile, (uint8_t*)marks_of(v0), tid);
    __syncthreads();
    for (int32_t v = v0; v < v1; ++v) {
      const int cur = (v - v0) & 1;
      if (v + 1 < v1) {
        st.load(a, kvh, tile_of(keys, v + 1) * KT, q.len, page, tid);
        if (v + 2 < v1) page = page_at(v + 2);
      }
      take_tile<T, DP, KT>(a, r, s_tile[cur], s_tile[cur] + kTile, marks_of(v), tile_of(keys, v) * KT);
      if (v + 1 < v1) st.write(s_tile[cur ^ 1], s_tile[cur ^ 1] + kTile, (uint8_t*)marks_of(v + 1), tid);
      __syncthreads();
    }
  }
  const int32_t row = base + 32 * wave + (lane & 31);
  const int h = lane >> 5;
  const float sum = r.sum + __shfl_xor(r.sum, 32);
  if (row < rows) {
    const int32_t i = row / a.group;
    const int head = kvh * a.group + (row - i * a.group);
    const int64_t t = q.t0 + i;
    const float vs = a.v_scale ? a.v_scale[kvh] : 1.0f;
    if (pieces == 1) {
      const bool none = r.pos < 0;
      const float by = vs / sum;
#pragma unroll
      for (int tt = 0; tt < DP / 32; ++tt)
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          const int d = 32 * tt + 8 * (j / 4) + 4 * h;
          if (d >= a.head_dim) continue;
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = none ? 0.0f : r.o[tt][j + e] * by;
          store4<T>((T*)a.out + t * a.o_token + (int64_t)head * a.o_head + d, x, a.o_vec);
        }
    } else {
      const int64_t at = part_row(a, chunk, t, head);
#pragma unroll
      for (int tt = 0; tt < DP / 32; ++tt)
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          const int d = 32 * tt + 8 * (j / 4) + 4 * h;
          if (d < a.head_dim) *(float4*)(a.part + at * a.head_dim + d) = float4{r.o[tt][j], r.o[tt][j + 1], r.o[tt][j + 2], r.o[tt][j + 3]};
        }
      if (h == 0) { a.part_ml[2 * at] = r.m; a.part_ml[2 * at + 1] = sum; }
    }
  }
  if (pieces > 1 && last_of(a.arrived_wide + (int64_t)tile * a.n_kv_head + kvh, (uint32_t)pieces, &s_flag)) join_rows<T>(a, q, kvh, base, n_row, pieces);
}

template <typename T, bool F8, int DP>
hipError_t launch_attention(const AttnArgs& a, hipStream_t s) {
  if (a.n_tile_wide > 0) {
    hipLaunchKernelGGL((attend_wide_kernel<T, F8, DP>), dim3((unsigned)a.n_tile_wide * a.n_kv_head, (unsigned)a.n_chunk_wide), dim3(64 * DYN_ATTN_WAVES_WIDE), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((attend_narrow_kernel<T, F8, DP>), dim3((unsigned)a.n_req * a.n_kv_head, (unsigned)a.n_chunk_narrow), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_type(const AttnArgs& a, hipStream_t s) {
  if (a.cache_type == DYN_T_E4M3) return a.head_dim <= 64 ? launch_attention<T, true, 64>(a, s) : launch_attention<T, true, 128>(a, s);
  return a.head_dim <= 64 ? launch_attention<T, false, 64>(a, s) : launch_attention<T, false, 128>(a, s);
}

}  // namespace

hipError_t dyn_launch_paged_attention(const AttnArgs& a, hipStream_t s) {
  DynTimed timed(DYN_K_ATTENTION, s);
  return a.type == DYN_T_BF16 ? launch_type<__bf16>(a, s) : launch_type<_Float16>(a, s);
}
