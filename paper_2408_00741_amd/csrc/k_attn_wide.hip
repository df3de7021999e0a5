// Attention for requests of many rows (new tokens x query heads of a key head): chunks of prompts.
#include "dyn_attn.h"

namespace {

__device__ __forceinline__ f32x16 mfma(x8<__bf16> a, x8<__bf16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma(x8<_Float16> a, x8<_Float16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

constexpr int KT = DYN_ATTN_KEYS_WIDE;

// Where 8 elements (16 bytes) of a tile lie in LDS, in units of 16 bytes: rows one after the other, the position in the row turned by the row so that the
// 16 lanes of a read hit all 64 banks: 16 keys' same elements of K, 4 keys' 32 neighbouring elements of V.  (Heads of 96 have the rows of 128.)  A step of the
// products then changes bits of the position that the key does not add to: one exclusive or makes its address.
template <int DP>
constexpr int kRow = DP <= 64 ? 8 : 16;
template <int DP>
__device__ __forceinline__ int k_at(int key, int c8) {
  return DP > 64 ? key * 16 + (c8 ^ (key & 15)) : key * 8 + (c8 ^ ((key >> 1) & 7));
}
template <int DP>
__device__ __forceinline__ int v_at(int key, int c8) {
  return DP > 64 ? key * 16 + (c8 ^ ((key & 3) << 2)) : key * 8 + (c8 ^ (((key >> 1) & 1) << 2));
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

// Row n (of the first product's left operand) of 32 keys is key swap23(n): bits 2 and 3 swapped.
__device__ __forceinline__ int swap23(int n) { return (n & 0x13) | ((n & 4) << 1) | ((n & 8) >> 1); }

// LDS by its byte address: the tiles begin at multiples of 256 bytes, so that the exclusive or of a step can be taken in the address itself.
typedef const __attribute__((address_space(3))) u32x4* LdsRead;
__device__ __forceinline__ uint32_t lds_address(const u32x4* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) u32x4*)p; }

// S^T of a tile whose keys are in LDS.
template <typename T, int DP>
__device__ __forceinline__ void scores(const Rows<T, DP>& r, const u32x4* lds_k, f32x16* s) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const uint32_t at = anew(16 * k_at<DP>(swap23(lane & 31), h)) + lds_address(lds_k);      // k_at(32 mt + .., 2 d + h) is (at ^ 32 d bytes) + 32 mt rows
#pragma unroll
  for (int mt = 0; mt < KT / 32; ++mt) {
    f32x16 acc = {};
#pragma unroll
    for (int d = 0; d < DP / 16; ++d) acc = mfma(__builtin_bit_cast(x8<T>, ((LdsRead)(uintptr_t)(at ^ 32 * d))[32 * mt * kRow<DP>]), r.q[d], acc);
    s[mt] = acc;
  }
}

// The rest of a tile: from the scores to the weighted sum of the values in LDS (v_at).  `key0`: the first key's position; `hidden`: some row does
// not see all of its keys; `marked`: `marks` has two bits of every value (take_out).
template <typename T, int DP>
__device__ __forceinline__ void weigh(const AttnArgs& a, Rows<T, DP>& r, f32x16* s, const u32x4* lds_v, bool hidden, bool marked, const uint32_t* marks, int32_t key0) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  // register i of s[mt] is key 32 mt + 16 (i / 8) + 8 h + i % 8.  What a row does not see scores -inf: weight 0 below, whatever the reference.
  if (hidden) {
    const int32_t mine = key0 + 8 * anew(h), from = a.window > 0 ? r.low - mine : -1, upto = r.pos - mine;      // seen: from < key <= upto, and the first tokens
    const uint32_t width = (uint32_t)max(upto - from, 0);
    const int32_t sinks = a.window > 0 ? min(a.n_sink - mine, upto + 1) : -1;
#pragma unroll
    for (int mt = 0; mt < KT / 32; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int32_t at = 32 * mt + 16 * (i / 8) + i % 8;
        s[mt][i] = (uint32_t)(at - 1 - from) < width || at < sinks ? s[mt][i] : -INFINITY;
        if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);
      }
  }
  float top = -INFINITY;
#pragma unroll
  for (int mt = 0; mt < KT / 32; ++mt)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[mt][i]);
  top = max_across_32(top);
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

  // V^T: lane group lane / 16 has elements 16 (group % 2) + .. of keys 8 (group / 2) + ..
  const int g16 = lane >> 4, i16 = lane & 15;
  const uint32_t at = anew(16 * v_at<DP>(8 * (g16 >> 1) + (i16 >> 2), 2 * (g16 & 1) + ((i16 & 3) >> 1)) + 8 * (i16 & 1)) + lds_address(lds_v);      // v_at(16 st + .., 4 t + ..) is (at ^ 64 t bytes) + 16 st rows
#pragma unroll
  for (int st = 0; st < KT / 16; ++st)
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) {
      const LdsRead v = (LdsRead)(uintptr_t)(at ^ 64 * t) + 16 * st * kRow<DP>;
      r.o[t] = mfma(__builtin_bit_cast(x8<T>, read_values(v, v + 4 * kRow<DP>)), p[st], r.o[t]);
    }
  // values that are not finite were taken out and marked: they go to the rows that see their keys.
  if (marked) {
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
            r.o[t][i] += sees ? marked_value(up, down, bit) : 0.0f;
          }
        }
      }
    }
  }
}

// Loads one wave's rows: rows base .. base + 31 of the request's `rows` for key head kvh.
template <typename T, int DP>
__device__ __forceinline__ void load_rows(const AttnArgs& a, const Request& q, int kvh, int32_t base, int32_t rows, Rows<T, DP>& r) {
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int32_t row = base + (lane & 31);
  const bool in = row < rows;
  const int32_t i = (in ? row : base) / a.group, g = (in ? row : base) - i * a.group;
  const float factor = factor_of(a, kvh);
  r.c = size_of(factor);
  const T* src = (const T*)a.q + (int64_t)(q.t0 + i) * a.q_token + (int64_t)(kvh * a.group + g) * a.q_head;
#pragma unroll
  for (int d = 0; d < DP / 16; ++d) r.q[d] = load_query<T>(a, src + 16 * d + 8 * h, in && 16 * d < a.head_dim, factor < 0.0f ? 0x80008000u : 0u);
  r.pos = in ? q.len - q.n + i : -1;
  r.low = a.window > 0 ? r.pos - a.window : -1;
  r.first = q.len - q.n + base / a.group;
  r.last = q.len - q.n + (min(base + 31, rows - 1)) / a.group;
  r.m = -INFINITY;
  r.sum = 0.0f;
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) r.o[t] = f32x16{};
}

// The part of a tile of keys or values that a wave carries from the cache to LDS: 16 neighbouring rows, which lie in one page of 16 tokens and more; a lane has pieces of
// 16 bytes, whole rows by neighbouring lanes.
constexpr int kWaveRows = KT / DYN_ATTN_WAVES_WIDE;
static_assert(kWaveRows == 16, "by_sixteen");
template <typename T, bool F8, int DP>
struct Stage {
  static constexpr int kPerRow = F8 ? kRow<DP> / 2 : kRow<DP>, kRows = 64 / kPerRow, kEach = kWaveRows / kRows;
  u32x4 x[kEach];
  static __device__ __forceinline__ int first_row(int wave, int i) { return wave * kWaveRows + i * kRows; }
  // `at`: where the wave's first row begins in the cache (by_sixteen), in bytes.  Keys beyond the request's last one are read as the last one (no row sees
  // them), pieces beyond the head's end as its first.
  __device__ __forceinline__ void load(const AttnArgs& a, const void* cache, int kvh, int b, int32_t key0, int32_t len, int wave, int64_t at, bool* bad) {
    const int row_bytes = a.head_dim * (F8 ? 1 : 2), lane = threadIdx.x & 63;
    if (by_sixteen(a, key0, KT, len)) {
      const int c = lane % kPerRow * 16;
      const uint32_t mine = lane / kPerRow * row_bytes + (c < row_bytes ? c : 0);
#pragma unroll
      for (int i = 0; i < kEach; ++i) x[i] = *(const u32x4*)((const char*)cache + at + i * kRows * row_bytes + mine);
    } else {
      const int l = anew(lane), c = l % kPerRow * 16, off = c < row_bytes ? c : 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int32_t key = min(key0 + first_row(wave, i) + l / kPerRow, len - 1);
        x[i] = *(const u32x4*)((const char*)cache + row_at(a, kvh, key, page_of(a, b, key, bad)) + off);
      }
    }
  }
  __device__ __forceinline__ void write_keys(const AttnArgs& a, u32x4* lds, int wave) {
    const int lane = threadIdx.x & 63, c = lane % kPerRow;
    if (a.head_dim < 8 * kRow<DP>) {        // beyond the head's end: zeros, as in the queries
      const bool in = c * 16 < a.head_dim * (F8 ? 1 : 2);
#pragma unroll
      for (int i = 0; i < kEach; ++i) x[i] = in ? x[i] : u32x4{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int row = first_row(wave, i) + lane / kPerRow;
#pragma unroll
      for (int e = 0; e < (F8 ? 2 : 1); ++e) lds[k_at<DP>(row, F8 ? 2 * c + e : c)] = F8 ? widen(T{}, x[i][2 * e], x[i][2 * e + 1]) : x[i];
    }
  }
  __device__ __forceinline__ void write_values(u32x4* lds, bool mark, uint8_t* marks, int wave) {
    const int lane = threadIdx.x & 63, c = lane % kPerRow;
    if (c >= DP / (F8 ? 16 : 8)) return;    // heads of 96: the rest of the row is not read
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int row = first_row(wave, i) + lane / kPerRow;
#pragma unroll
      for (int e = 0; e < (F8 ? 2 : 1); ++e) {
        const int c8 = F8 ? 2 * c + e : c;
        u32x4 v = F8 ? widen(T{}, x[i][2 * e], x[i][2 * e + 1]) : x[i];
        if (mark) v = take_out<T>(v, marks + row * (DP / 8) + c8, marks + (KT + row) * (DP / 8) + c8);
        lds[v_at<DP>(row, c8)] = v;
      }
    }
  }
};

// The same straight into LDS, for 16-bit heads that fill their rows (64, 96 or 128 wide): no registers, no second way.  A load puts its 64 lanes' pieces one after the other,
// so that a lane takes the piece of its row that belongs where it writes.
template <typename T, int DP>
struct Direct {
  static constexpr int kPerRow = kRow<DP>, kRows = 64 / kPerRow, kEach = kWaveRows / kRows;
  // the piece of its row that lane `lane` takes of the wave's load i: of keys, of values (the same for all loads: their rows are multiples of 4 apart)
  static __device__ __forceinline__ int key_piece(int i, int lane) { return k_at<DP>(i * kRows + lane / kPerRow, lane % kPerRow) % kPerRow; }
  static __device__ __forceinline__ int value_piece(int lane) { return v_at<DP>(lane / kPerRow, lane % kPerRow) % kPerRow; }
  template <bool KEYS>
  static __device__ __forceinline__ void load(const AttnArgs& a, u32x4* lds, int kvh, int b, int32_t key0, int32_t len, int wave, int64_t at, bool* bad) {
    typedef const __attribute__((address_space(1))) uint32_t* from;
    typedef __attribute__((address_space(3))) uint32_t* to;
    const int lane = threadIdx.x & 63;
    const char* cache = (const char*)(KEYS ? a.k_cache : a.v_cache);
    u32x4* here = lds + wave * kWaveRows * kPerRow;
    if (by_sixteen(a, key0, KT, len)) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int piece = KEYS ? key_piece(i, lane) : value_piece(lane);
        const uint32_t mine = (i * kRows + lane / kPerRow) * (DP * 2) + piece * 16;
        if (kPerRow * 8 == DP || piece * 8 < DP)             // heads of 96: the rest of the row is not read
          __builtin_amdgcn_global_load_lds((from)(cache + at + mine), (to)(here + i * 64), 16, 0, 0);
      }
    } else {
      const int l = anew(lane);
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int piece = KEYS ? key_piece(i, l) : value_piece(l);
        const int32_t key = min(key0 + wave * kWaveRows + i * kRows + l / kPerRow, len - 1);
        const char* row = cache + row_at(a, kvh, key, page_of(a, b, key, bad));
        if (kPerRow * 8 == DP || piece * 8 < DP) __builtin_amdgcn_global_load_lds((from)(row + piece * 16), (to)(here + i * 64), 16, 0, 0);
      }
    }
  }
  // Takes the values that are not finite out of a tile in LDS.
  static __device__ __forceinline__ void mark_values(u32x4* lds, uint8_t* marks, int wave) {
    const int lane = anew(threadIdx.x & 63), c = value_piece(lane);
    if (c * 8 >= DP) return;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int row = wave * kWaveRows + i * kRows + lane / kPerRow, at = (wave * kWaveRows + i * kRows) * kPerRow + lane;
      lds[at] = take_out<T>(lds[at], marks + row * (DP / 8) + c, marks + (KT + row) * (DP / 8) + c);
    }
  }
};

// Requests of more rows: a block has 32 rows for each of its waves, all waves read the same tiles of 64 keys from LDS, two tiles in turn, the next
// one's loads in flight while one is worked on.  Bound by the matrix instructions and the exponentials beside them.
template <typename T, bool F8, int DP, bool DIRECT>
__global__ __launch_bounds__(64 * DYN_ATTN_WAVES_WIDE, 2) void attend_wide_kernel(AttnArgs a) {
  constexpr int NW = DYN_ATTN_WAVES_WIDE, R = 32 * NW, kTile = KT * kRow<DP>;   // 16-byte pieces of K (or V) of a tile
  __shared__ __attribute__((aligned(256))) u32x4 s_tile[2][2 * kTile];
  __shared__ uint32_t s_marks[2][2 * KT * DP / 32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.n_kv_head, chunk = blockIdx.y;
  if (blockIdx.x == 0 && chunk == 0 && tid == 0) a.header->kind = DYN_WS_KIND_WORD;
  // row tiles are numbered so that request b's begin at cu[b] x group / R + b: the request of a tile follows from cu alone.  Later tiles have more
  // keys: they come first.
  const int32_t tile = a.n_tile_wide - 1 - blockIdx.x / a.n_kv_head;
  auto begin_of = [&](int b) { return (int64_t)min(max(a.cu[b], 0), a.n_token) * a.group / R + b; };
  const int b = last_request(a.n_req, [&](int b) { return begin_of(b) <= tile; });
  const Request q = request_of(a, b);
  const int64_t all_rows = (int64_t)q.n * a.group, base64 = ((int64_t)tile - begin_of(b)) * R;
  if (all_rows <= a.rows_narrow || base64 < 0 || base64 >= all_rows) return;
  const int32_t rows = (int32_t)all_rows, base = (int32_t)base64, n_row = min(R, rows - base);
  const int32_t first = q.len - q.n + base / a.group, last = q.len - q.n + (base + n_row - 1) / a.group;
  const Keys keys = last >= 0 ? keys_of<KT>(a, first, last) : Keys{0, 0, 0};
  const int pieces = pieces_of(keys, a.n_chunk_wide, a.tiles_wide);
  if (chunk >= pieces) return;
  const int32_t v0 = chunk * a.tiles_wide, v1 = chunk == a.n_chunk_wide - 1 ? keys.count : min(keys.count, v0 + a.tiles_wide);
  Rows<T, DP> r;
  const bool idle = base + 32 * wave >= rows;
  load_rows<T, DP>(a, q, kvh, idle ? 0 : base + 32 * wave, idle ? 0 : rows, r);
  if (idle) r.last = -1;
  bool bad = false;
  if (v0 < v1) {
    // where this wave's rows of the next tile begin; the table's entry is fetched a tile before
    int64_t next = 0;
    int32_t entry = 0;
    auto key_at = [&](int32_t v) { return min(tile_of(keys, min(v, v1 - 1)) * KT + wave * kWaveRows, q.len - 1); };
    auto fetch = [&](int32_t v) { entry = entry_of_all(a, b, key_at(v)); };
    auto find = [&](int32_t v) { next = row_at(a, kvh, key_at(v), inside(a, entry, &bad)); };
    // tiles [from, to) are seen in whole by all rows, of the block and of this wave (and others perhaps)
    auto whole = [&](int32_t lo, int32_t hi, int32_t* from, int32_t* to) {
      const int32_t shift = keys.first - keys.sink_tiles;              // of a tile's number and its keys, from the window on
      *from = a.window > 0 && hi >= a.window ? max((hi - a.window) / KT + 1 - shift, keys.sink_tiles) : 0;
      *to = max(lo + 1, 0) / KT - shift;
      if (*to < keys.sink_tiles) *to = 0;                              // the window itself begins in the first tokens
    };
    int32_t block_from, block_to, wave_from, wave_to;
    whole(first, last, &block_from, &block_to);
    whole(r.first, r.last, &wave_from, &wave_to);
    auto marked = [&](int32_t v) { return v < block_from || v >= block_to; };
    auto work = [&](int32_t v) {
      const u32x4* at = s_tile[(v - v0) & 1];
      const int32_t key0 = tile_of(keys, v) * KT;
      // none of this wave's rows sees a key of the tile: beyond the last row's, or before the first row's window and after the first tokens
      if (key0 <= r.last && !(a.window > 0 && key0 + KT - 1 <= r.first - a.window && key0 >= a.n_sink)) {
        f32x16 s[KT / 32];
        scores<T, DP>(r, at, s);
        weigh<T, DP>(a, r, s, at + kTile, v < wave_from || v >= wave_to, marked(v), s_marks[(v - v0) & 1], key0);
      }
    };
    if constexpr (DIRECT) {
      using D = Direct<T, DP>;
      auto load = [&](int32_t v) {
        u32x4* at = s_tile[(v - v0) & 1];
        D::template load<true>(a, at, kvh, b, tile_of(keys, v) * KT, q.len, wave, next, &bad);
        D::template load<false>(a, at + kTile, kvh, b, tile_of(keys, v) * KT, q.len, wave, next, &bad);
      };
      fetch(v0);
      find(v0);
      fetch(v0 + 1);
      load(v0);
      for (int32_t v = v0; v < v1; ++v) {
        __syncthreads();           // this tile is there, and all waves are through with the one before
        if (marked(v)) {
          D::mark_values(s_tile[(v - v0) & 1] + kTile, (uint8_t*)s_marks[(v - v0) & 1], wave);
          __syncthreads();
        }
        if (v + 1 < v1) {
          find(v + 1);
          fetch(v + 2);
          load(v + 1);
        }
        work(v);
      }
    } else {
      Stage<T, F8, DP> sk, sv;
      auto load = [&](int32_t v) {
        sk.load(a, a.k_cache, kvh, b, tile_of(keys, v) * KT, q.len, wave, next, &bad);
        sv.load(a, a.v_cache, kvh, b, tile_of(keys, v) * KT, q.len, wave, next, &bad);
      };
      auto write = [&](int32_t v) {
        u32x4* at = s_tile[(v - v0) & 1];
        sk.write_keys(a, at, wave);
        sv.write_values(at + kTile, marked(v), (uint8_t*)s_marks[(v - v0) & 1], wave);
      };
      fetch(v0);
      find(v0);
      fetch(v0 + 1);
      load(v0);
      write(v0);
      __syncthreads();
      for (int32_t v = v0; v < v1; ++v) {
        if (v + 1 < v1) {
          find(v + 1);
          fetch(v + 2);
          load(v + 1);
        }
        work(v);
        if (v + 1 < v1) write(v + 1);
        __syncthreads();
      }
    }
  }
  report(a, bad);
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
}


template <typename T, bool F8, int DP>
hipError_t launch(const AttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.n_tile_wide * a.n_kv_head, (unsigned)a.n_chunk_wide), block(64 * DYN_ATTN_WAVES_WIDE);
  if (!F8 && a.head_dim == DP) hipLaunchKernelGGL((attend_wide_kernel<T, F8, DP, !F8>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((attend_wide_kernel<T, F8, DP, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
template <typename T, bool F8>
hipError_t launch_dim(const AttnArgs& a, hipStream_t s) {   // heads are taken as 64, 96 or 128 wide, zeros beyond their end
  return a.head_dim <= 64 ? launch<T, F8, 64>(a, s) : a.head_dim <= 96 ? launch<T, F8, 96>(a, s) : launch<T, F8, 128>(a, s);
}
template <typename T>
hipError_t launch_type(const AttnArgs& a, hipStream_t s) { return a.cache_type == DYN_T_E4M3 ? launch_dim<T, true>(a, s) : launch_dim<T, false>(a, s); }

}  // namespace

hipError_t dyn_launch_attend_wide(const AttnArgs& a, hipStream_t s) { return a.type == DYN_T_BF16 ? launch_type<__bf16>(a, s) : launch_type<_Float16>(a, s); }
