// Gated feed-forward block over kept rows: argument checks, workspaces, choice of tiles, and the launches.
//
//   g = X Wg', u = X Wu', hidden = act(g) u, y = hidden Wd'
//   dhidden = dY Wd, dg = dhidden u act'(g), du = dhidden act(g), dX = dg Wg + du Wu, dWd = dY' hidden, dWg = dg' X, dWu = du' X
//
// 6 kept d F operations forward and 12 backward on the matrix cores; the rows that the mask drops are neither read nor multiplied.
// hidden, dg and du are rounded to the operands' type between the launches (they are operands of the next product); everything
// else stays in float until it is stored.
#include "../../include/sparse_block.h"
#include "ffn_params.hpp"
#include "rows.hpp"

#include <initializer_list>

namespace sc {

void note_hip_error(int32_t code);

enum : int32_t { kTypeF32 = SC_F32, kTypeF16 = SC_F16, kTypeBF16 = SC_BF16 };

static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
static int elem_bytes(int dtype) { return dtype == SC_F32 ? 4 : 2; }

static sc_status check_ffn(const sc_ffn_desc* d, int64_t kept) {
  if (!d) return SC_ERR_NULL;
  if (d->dtype != SC_F32 && d->dtype != SC_F16 && d->dtype != SC_BF16) return SC_ERR_UNSUPPORTED;
  if (d->activation < SC_ACT_SILU || d->activation > SC_ACT_GELU_TANH) return SC_ERR_UNSUPPORTED;
  const int32_t most = 1 << 20;
  if (d->d_in < 1 || d->d_hidden < 1 || d->d_out < 1 || d->d_in > most || d->d_hidden > most || d->d_out > most) return SC_ERR_BAD_SHAPE;
  if (kept < 0 || kept > 0x7fffffff - 4096) return SC_ERR_BAD_SHAPE;
  return SC_OK;
}

static hipError_t launch(int dtype, FfnProduct what, const FfnGemm& g, int tile, bool aligned, hipStream_t s) {
  switch (dtype) {
    case SC_BF16: return ffn_launch_bf16(what, g, tile, aligned, s);
    case SC_F16: return ffn_launch_f16(what, g, tile, aligned, s);
    default: return ffn_launch_f32(what, g, tile, aligned, s);
  }
}

constexpr int64_t kFewRows = 64;

static hipError_t launch_forward(int dtype, FfnProduct what, const FfnGemm& g, int tile, bool aligned, hipStream_t s) {
  if (g.m > kFewRows) return launch(dtype, what, g, tile, aligned, s);
  switch (dtype) {
    case SC_BF16: return ffn_few_bf16(what == kFfnUp, g, aligned, s);
    case SC_F16: return ffn_few_f16(what == kFfnUp, g, aligned, s);
    default: return ffn_few_f32(what == kFfnUp, g, aligned, s);
  }
}

static bool whole_groups(const sc_ffn_desc& d) {
  const int v = 16 / elem_bytes(d.dtype);
  return d.d_in % v == 0 && d.d_hidden % v == 0 && d.d_out % v == 0;
}

// Tiles of 256 x 256 where they fill the chip, 128 x 128 otherwise.
static int pick_tile(int64_t m, int64_t cols, int batch) {
  const int64_t big = ((m + 255) / 256) * ((cols + 255) / 256) * batch;
  return big >= 192 ? 1 : 0;
}

// Parts of the contraction over rows: a weight gradient has few tiles and many rows.  Every part leaves its sums in float.
static int pick_splits(int64_t m, int64_t n, int batch, int tile, int64_t kept, int dtype) {
  const int edge = tile == 1 ? 256 : 128, bk = dtype == SC_F32 ? 32 : 64;
  const int64_t tiles = ((m + edge - 1) / edge) * ((n + edge - 1) / edge) * batch;
  const int64_t wanted = (tile == 1 ? 256 : 512) / tiles, most = ((kept + bk - 1) / bk) / 8;
  const int64_t splits = wanted < most ? wanted : most;
  return splits < 1 ? 1 : splits > 64 ? 64 : (int)splits;
}

static size_t partial_bytes(const sc_ffn_desc& d, int64_t kept) {
  size_t most = 0;
  const int tile_in = pick_tile(d.d_hidden, d.d_in, 2), tile_out = pick_tile(d.d_out, d.d_hidden, 1);
  const int s_in = pick_splits(d.d_hidden, d.d_in, 2, tile_in, kept, d.dtype);
  const int s_out = pick_splits(d.d_out, d.d_hidden, 1, tile_out, kept, d.dtype);
  if (s_in > 1) most = (size_t)2 * s_in * d.d_hidden * d.d_in * 4;
  if (s_out > 1 && (size_t)s_out * d.d_out * d.d_hidden * 4 > most) most = (size_t)s_out * d.d_out * d.d_hidden * 4;
  return up256(most);
}

// sums of the parts, in order; batch results of `count` values each
template <typename T>
__global__ __launch_bounds__(256) void ffn_sum_parts_kernel(const float* __restrict__ partial, T* c0, T* c1, int64_t count,
                                                            int splits) {
  const int z = blockIdx.y;
  T* c = z ? c1 : c0;
  const float* p = partial + (int64_t)z * splits * count;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
    float v = 0.0f;
    for (int s = 0; s < splits; ++s) v += p[(int64_t)s * count + i];
    c[i] = (T)v;
  }
}

static hipError_t sum_parts(int dtype, const FfnGemm& g, hipStream_t s) {
  const int64_t count = (int64_t)g.m * g.n;
  const int64_t want = (count + 255) / 256;
  const dim3 grid((unsigned)(want < 4096 ? want : 4096), g.batch);
  if (dtype == SC_BF16)
    ffn_sum_parts_kernel<__bf16><<<grid, dim3(256), 0, s>>>(g.partial, (__bf16*)g.c[0], (__bf16*)g.c[1], count, g.splits);
  else if (dtype == SC_F16)
    ffn_sum_parts_kernel<_Float16><<<grid, dim3(256), 0, s>>>(g.partial, (_Float16*)g.c[0], (_Float16*)g.c[1], count, g.splits);
  else
    ffn_sum_parts_kernel<float><<<grid, dim3(256), 0, s>>>(g.partial, (float*)g.c[0], (float*)g.c[1], count, g.splits);
  return hipGetLastError();
}

__global__ __launch_bounds__(256) void ffn_zero_kernel(uint16_t* out, int64_t count) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) out[i] = 0;
}
static hipError_t zero(void* out, size_t bytes, hipStream_t s) {
  if (!out || bytes == 0) return hipSuccess;
  const int64_t want = (int64_t)(bytes / 2 + 255) / 256;
  ffn_zero_kernel<<<dim3((unsigned)(want < 2048 ? want : 2048)), dim3(256), 0, s>>>((uint16_t*)out, (int64_t)(bytes / 2));
  return hipGetLastError();
}

// the checks that run and backward share
static sc_status check_call(const sc_ffn_desc* d, int64_t m, const sc_rows* rows, int32_t x_rows, int32_t y_rows, int64_t* kept) {
  sc_status st = check_ffn(d, m);
  if (st != SC_OK) return st;
  if ((x_rows != SC_ROWS_DENSE && x_rows != SC_ROWS_COMPACT) || (y_rows != SC_ROWS_DENSE && y_rows != SC_ROWS_COMPACT))
    return SC_ERR_UNSUPPORTED;
  if (rows && rows->rows != m) return SC_ERR_BAD_SHAPE;
  *kept = rows ? rows->kept : m;
  return SC_OK;
}

static bool misaligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if ((uintptr_t)p & 15) return true;
  return false;
}

// the list of kept rows, for a tensor in the dense layout; null where the rows are those of the tensor
static const int32_t* map_of(const sc_rows* rows, int32_t format) {
  return rows && format == SC_ROWS_DENSE && rows->kept != rows->rows ? rows->row_idx : nullptr;
}

static sc_status failed(hipError_t e) {
  note_hip_error((int32_t)e);
  return SC_ERR_HIP;
}

static FfnGemm gemm_of(int64_t m, int64_t n, int64_t k) {
  FfnGemm g = {};
  g.m = (int32_t)m;
  g.n = (int32_t)n;
  g.k = (int32_t)k;
  g.segments = g.batch = g.splits = 1;
  return g;
}

}  // namespace sc

extern "C" {

sc_status sparse_ffn_workspace_bytes(const sc_ffn_desc* desc, int64_t kept, int32_t training, size_t* bytes) {
  if (!bytes) return SC_ERR_NULL;
  *bytes = 0;
  const sc_status st = sc::check_ffn(desc, kept);
  if (st != SC_OK) return st;
  const size_t hidden = sc::up256((size_t)kept * desc->d_hidden * sc::elem_bytes(desc->dtype));
  *bytes = 256 + (training ? 2 * hidden + sc::partial_bytes(*desc, kept) : hidden);
  return SC_OK;
}

sc_status sparse_ffn_run(const sc_ffn_desc* desc, int64_t m, const sc_rows* rows, const void* x_dev, int32_t x_rows,
                         const void* w_gate_dev, const void* w_up_dev, const void* w_down_dev, void* y_dev, int32_t y_rows,
                         void* saved_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  int64_t kept = 0;
  sc_status st = sc::check_call(desc, m, rows, x_rows, y_rows, &kept);
  if (st != SC_OK) return st;
  if (!w_gate_dev || !w_up_dev || !w_down_dev || !workspace_dev || (m > 0 && !y_dev && (kept > 0 || y_rows == SC_ROWS_DENSE)) ||
      (kept > 0 && !x_dev))
    return SC_ERR_NULL;
  size_t need = 0;
  sparse_ffn_workspace_bytes(desc, kept, 0, &need);
  if (!saved_dev && workspace_bytes < need) return SC_ERR_WORKSPACE;
  if (sc::misaligned({x_dev, w_gate_dev, w_up_dev, w_down_dev, y_dev, saved_dev, workspace_dev})) return SC_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int eb = sc::elem_bytes(desc->dtype);
  const bool aligned = sc::whole_groups(*desc);
  hipError_t e = hipSuccess;
  if (y_rows == SC_ROWS_DENSE) e = sc::rows_zero_dropped(rows, (int64_t)desc->d_out * eb, y_dev, s);
  if (e != hipSuccess) return sc::failed(e);
  if (kept == 0) return SC_OK;
  void* hidden = saved_dev ? static_cast<char*>(saved_dev) + (size_t)2 * kept * desc->d_hidden * eb : workspace_dev;

  sc::FfnGemm up = sc::gemm_of(kept, desc->d_hidden, desc->d_in);
  up.p[0] = x_dev;
  up.ldp = up.ldq = desc->d_in;
  up.p_rows = sc::map_of(rows, x_rows);
  up.q[0] = w_gate_dev;
  up.q[1] = w_up_dev;
  up.c[0] = hidden;
  up.ldc = desc->d_hidden;
  up.saved = saved_dev;
  up.activation = desc->activation;
  e = sc::launch_forward(desc->dtype, sc::kFfnUp, up, sc::pick_tile(kept, 2 * (int64_t)desc->d_hidden, 1), aligned, s);
  if (e != hipSuccess) return sc::failed(e);

  sc::FfnGemm down = sc::gemm_of(kept, desc->d_out, desc->d_hidden);
  down.p[0] = hidden;
  down.q[0] = w_down_dev;
  down.ldp = down.ldq = desc->d_hidden;
  down.c[0] = y_dev;
  down.ldc = desc->d_out;
  down.c_rows = sc::map_of(rows, y_rows);
  e = sc::launch_forward(desc->dtype, sc::kFfnDown, down, sc::pick_tile(kept, desc->d_out, 1), aligned, s);
  return e == hipSuccess ? SC_OK : sc::failed(e);
}

sc_status sparse_ffn_backward(const sc_ffn_desc* desc, int64_t m, const sc_rows* rows, const void* x_dev, int32_t x_rows,
                              const void* w_gate_dev, const void* w_up_dev, const void* w_down_dev, const void* saved_dev,
                              const void* dy_dev, int32_t y_rows, void* dx_dev, void* dw_gate_dev, void* dw_up_dev,
                              void* dw_down_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  int64_t kept = 0;
  sc_status st = sc::check_call(desc, m, rows, x_rows, y_rows, &kept);
  if (st != SC_OK) return st;
  const bool weights = dw_gate_dev || dw_up_dev || dw_down_dev;
  if (weights && !(dw_gate_dev && dw_up_dev && dw_down_dev)) return SC_ERR_NULL;
  if (!w_gate_dev || !w_up_dev || !w_down_dev || !workspace_dev || (kept > 0 && (!x_dev || !saved_dev || !dy_dev))) return SC_ERR_NULL;
  size_t need = 0;
  sparse_ffn_workspace_bytes(desc, kept, 1, &need);
  if (workspace_bytes < need) return SC_ERR_WORKSPACE;
  if (sc::misaligned({x_dev, w_gate_dev, w_up_dev, w_down_dev, saved_dev, dy_dev, dx_dev, dw_gate_dev, dw_up_dev, dw_down_dev,
                      workspace_dev}))
    return SC_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int eb = sc::elem_bytes(desc->dtype);
  const int64_t d_in = desc->d_in, d_hidden = desc->d_hidden, d_out = desc->d_out;
  const bool aligned = sc::whole_groups(*desc);
  hipError_t e = hipSuccess;
  if (dx_dev && x_rows == SC_ROWS_DENSE) e = sc::rows_zero_dropped(rows, d_in * eb, dx_dev, s);
  if (e != hipSuccess) return sc::failed(e);
  if (kept == 0) {
    if (e == hipSuccess) e = sc::zero(dw_gate_dev, (size_t)d_hidden * d_in * eb, s);
    if (e == hipSuccess) e = sc::zero(dw_up_dev, (size_t)d_hidden * d_in * eb, s);
    if (e == hipSuccess) e = sc::zero(dw_down_dev, (size_t)d_out * d_hidden * eb, s);
    return e == hipSuccess ? SC_OK : sc::failed(e);
  }
  char* const w = static_cast<char*>(workspace_dev);
  const size_t hidden_bytes = (size_t)kept * d_hidden * eb;
  void* const dg = w;
  void* const du = w + sc::up256(hidden_bytes);
  float* const partial = reinterpret_cast<float*>(w + 2 * sc::up256(hidden_bytes));

  sc::FfnGemm gate = sc::gemm_of(kept, d_hidden, d_out);       // dhidden = dY Wd, then dg and du
  gate.p[0] = dy_dev;
  gate.ldp = d_out;
  gate.p_rows = sc::map_of(rows, y_rows);
  gate.q[0] = w_down_dev;
  gate.ldq = d_hidden;
  gate.saved = const_cast<void*>(saved_dev);
  gate.c[0] = dg;
  gate.c[1] = du;
  gate.ldc = d_hidden;
  gate.activation = desc->activation;
  e = sc::launch(desc->dtype, sc::kFfnGateGrad, gate, sc::pick_tile(kept, d_hidden, 1), aligned, s);
  if (e != hipSuccess) return sc::failed(e);

  if (dx_dev) {
    sc::FfnGemm in = sc::gemm_of(kept, d_in, d_hidden);
    in.segments = 2;
    in.p[0] = dg;
    in.p[1] = du;
    in.ldp = d_hidden;
    in.q[0] = w_gate_dev;
    in.q[1] = w_up_dev;
    in.ldq = d_in;
    in.c[0] = dx_dev;
    in.ldc = d_in;
    in.c_rows = sc::map_of(rows, x_rows);
    e = sc::launch(desc->dtype, sc::kFfnInGrad, in, sc::pick_tile(kept, d_in, 1), aligned, s);
    if (e != hipSuccess) return sc::failed(e);
  }
  if (weights) {
    sc::FfnGemm in = sc::gemm_of(d_hidden, d_in, kept);        // dWg = dg' X, dWu = du' X
    in.batch = 2;
    in.p[0] = dg;
    in.p[1] = du;
    in.ldp = d_hidden;
    in.q[0] = x_dev;
    in.ldq = d_in;
    in.q_rows = sc::map_of(rows, x_rows);
    in.c[0] = dw_gate_dev;
    in.c[1] = dw_up_dev;
    in.ldc = d_in;
    in.partial = partial;
    const int tile_in = sc::pick_tile(d_hidden, d_in, 2);
    in.splits = sc::pick_splits(d_hidden, d_in, 2, tile_in, kept, desc->dtype);
    e = sc::launch(desc->dtype, sc::kFfnWGrad, in, tile_in, aligned, s);
    if (e == hipSuccess && in.splits > 1) e = sc::sum_parts(desc->dtype, in, s);
    if (e != hipSuccess) return sc::failed(e);

    sc::FfnGemm out = sc::gemm_of(d_out, d_hidden, kept);      // dWd = dY' hidden
    out.p[0] = dy_dev;
    out.ldp = d_out;
    out.p_rows = sc::map_of(rows, y_rows);
    out.q[0] = static_cast<const char*>(saved_dev) + 2 * hidden_bytes;
    out.ldq = d_hidden;
    out.c[0] = dw_down_dev;
    out.ldc = d_hidden;
    out.partial = partial;
    const int tile_out = sc::pick_tile(d_out, d_hidden, 1);
    out.splits = sc::pick_splits(d_out, d_hidden, 1, tile_out, kept, desc->dtype);
    e = sc::launch(desc->dtype, sc::kFfnWGrad, out, tile_out, aligned, s);
    if (e == hipSuccess && out.splits > 1) e = sc::sum_parts(desc->dtype, out, s);
    if (e != hipSuccess) return sc::failed(e);
  }
  return SC_OK;
}

}  // extern "C"
