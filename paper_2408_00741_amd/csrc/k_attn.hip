// Attention over the paged cache: the launches, and the kernel that joins the pieces of the wide kernel's rows.
#include "dyn_attn.h"

namespace {

// Joins the pieces of the wide kernel's rows, a wave for each row.  The sum goes in the order of the pieces: the same values on every run.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(AttnArgs a) {
  const int lane = threadIdx.x & 63, heads = a.n_kv_head * a.group;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= (int64_t)a.n_token * heads) return;
  const int32_t t = (int32_t)(row / heads);
  const int head = (int)(row - (int64_t)t * heads), kvh = head / a.group;
  const int b = last_request(a.n_req, [&](int b) { return a.cu[b] <= t; });
  const Request q = request_of(a, b);
  if (t < q.t0 || t >= q.t0 + q.n) return;
  const int64_t rows = (int64_t)q.n * a.group;
  const int32_t pos = q.len - q.n + (t - q.t0);
  if (rows <= a.rows_narrow) return;
  constexpr int R = 32 * DYN_ATTN_WAVES_WIDE;
  const int64_t base = ((int64_t)(t - q.t0) * a.group + (head - kvh * a.group)) / R * R;
  const int32_t first = q.len - q.n + (int32_t)(base / a.group), last = q.len - q.n + (int32_t)((min(base + R, rows) - 1) / a.group);
  const int pieces = last >= 0 ? pieces_of(keys_of<DYN_ATTN_KEYS_WIDE>(a, first, last), a.n_chunk_wide, a.tiles_wide) : 1;
  if (pieces == 1) return;
  const float vs = a.v_scale ? a.v_scale[kvh] : 1.0f, c = size_of(factor_of(a, kvh));
  const int64_t step = (int64_t)a.n_token * heads;
  float m = -INFINITY;
  for (int p = lane; p < pieces; p += 64) m = fmaxf(m, a.part_ml[2 * (p * step + row)]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  float sum = 0.0f, x = 0.0f, y = 0.0f;
  const int at = 2 * lane;
  const bool in = at < a.head_dim;
  for (int p0 = 0; p0 < pieces; p0 += 8) {
    float2 ml[8], v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = min(p0 + i, pieces - 1) * step + row;
      ml[i] = *(const float2*)(a.part_ml + 2 * r);
      v[i] = *(const float2*)(a.part + r * a.head_dim + (in ? at : 0));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (p0 + i >= pieces || (ml[i].x == -INFINITY && ml[i].y == 0.0f)) continue;     // no weight in this piece
      const float f = ml[i].x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((ml[i].x - m) * c);
      sum = __builtin_fmaf(ml[i].y, f, sum);
      x = __builtin_fmaf(v[i].x, f, x);
      y = __builtin_fmaf(v[i].y, f, y);
    }
  }
  if (!in) return;
  T* to = (T*)a.out + t * a.o_token + head * a.o_head + at;
  const float by = vs / sum;
  to[0] = (T)(pos < 0 ? 0.0f : x * by);
  to[1] = (T)(pos < 0 ? 0.0f : y * by);
}

}  // namespace

hipError_t dyn_launch_paged_attention(const AttnArgs& a, hipStream_t s) {
  DynTimed timed(DYN_K_ATTENTION, s);
  hipError_t e = hipSuccess;
  if (a.n_tile_wide > 0 && (e = dyn_launch_attend_wide(a, s)) != hipSuccess) return e;
  if (a.rows_narrow >= a.group && (e = dyn_launch_attend_narrow(a, s)) != hipSuccess) return e;
  if (a.n_chunk_wide == 1) return e;
  const dim3 grid((unsigned)(((int64_t)a.n_token * a.n_kv_head * a.group + 3) / 4));
  if (a.type == DYN_T_BF16) hipLaunchKernelGGL((join_kernel<__bf16>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((join_kernel<_Float16>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
