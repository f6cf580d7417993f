// Gated feed-forward block over kept rows: argument checks, workspaces, choice of tiles, and the launches.
//
//   g = X Wg', u = X Wu', hidden = act(g) u, y = hidden Wd'
//   dhidden = dY Wd, dg = dhidden u act'(g), du = dhidden act(g), dX = dg Wg + du Wu, dWd = dY' hidden, dWg = dg' X, dWu = du' X
//
// 6 kept d F operations forward and 12 backward on the matrix cores; the rows that the mask drops are neither read nor multiplied.
// hidden, dg and du are rounded to the operands' type between the launches (they are operands of the next product); everything
// else stays in float until it is stored.
#include "../../include/sparse_block.h"
#include "ffn_act.hpp"
#include "ffn_params.hpp"
#include "ffn_saved.hpp"
#include "mma_common.hpp"
#include "rows.hpp"

#include <algorithm>
#include <initializer_list>

namespace sc {

void note_hip_error(int32_t code);

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

static hipError_t launch(int dtype, FfnProduct what, const FfnGemm& g, int tile, bool whole, hipStream_t s) {
  switch (dtype) {
    case SC_BF16: return ffn_launch_bf16(what, g, tile, whole, s);
    case SC_F16: return ffn_launch_f16(what, g, tile, whole, s);
    default: return ffn_launch_f32(what, g, tile, whole, s);
  }
}

constexpr int64_t kFewRows = 64;

// entries from row to row of an operand: whole 16-byte groups
static int64_t pitch_of(int64_t entries, int dtype) {
  const int64_t group = 16 / elem_bytes(dtype);
  return (entries + group - 1) / group * group;
}
static bool whole_rows(const sc_ffn_desc& d) { return (d.d_in | d.d_hidden | d.d_out) * elem_bytes(d.dtype) % 16 == 0; }

// Operands whose rows are not whole 16-byte groups are copied first, kept rows alone, with zeros up to the next whole group: the products
// then load straight into LDS and have no ends to look after.  5 000 x 423 -> 2 809 in bf16, forward and backward, takes
// 310 us (424 -> 2 808: 248), 699 where rows went through registers into LDS.
constexpr int kMostCopies = 5;
struct FfnCopies {
  struct One {
    const void* src;
    void* dst;
    const int32_t* rows;      // row of src that row i stands for; null: i
    uint32_t cols, groups;    // entries a row, 16-byte groups a row of dst
    int64_t first;            // group of the launch that is dst's first
  } one[kMostCopies];
  int32_t count, elem;
  int64_t groups;
};
template <typename T> __global__ __launch_bounds__(256) void ffn_copy_kernel(const FfnCopies c) {
  constexpr uint32_t V = 16 / sizeof(T);
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= c.groups) return;
  int which = 0;
  while (which + 1 < c.count && at >= c.one[which + 1].first) ++which;
  const FfnCopies::One& o = c.one[which];
  const int64_t local = at - o.first;
  const int64_t row = local >> 32 ? local / o.groups : (uint32_t)local / o.groups;
  const uint32_t col = (uint32_t)(local - row * o.groups) * V;
  const T* src = static_cast<const T*>(o.src) + (o.rows ? (int64_t)o.rows[row] : row) * o.cols + col;
  T v[V];
#pragma unroll
  for (uint32_t e = 0; e < V; ++e) v[e] = T(0);
  if (col + V <= o.cols) {
    __builtin_memcpy(v, src, 16);
  } else {
#pragma unroll
    for (uint32_t e = 0; e < V; ++e)
      if (col + e < o.cols) v[e] = src[e];
  }
  __builtin_memcpy(__builtin_assume_aligned(static_cast<T*>(o.dst) + local * V, 16), v, 16);
}
struct Copies {
  FfnCopies c = {};
  char* at;
  explicit Copies(void* workspace, int dtype) : at(static_cast<char*>(workspace)) { c.elem = elem_bytes(dtype); }
  static size_t bytes(int64_t rows, int64_t cols, int dtype) { return up256((size_t)rows * pitch_of(cols, dtype) * elem_bytes(dtype)); }
  const void* add(const void* src, int64_t rows, int64_t cols, int dtype, const int32_t* list = nullptr) {
    const int64_t groups = pitch_of(cols, dtype) * c.elem / 16;
    c.one[c.count++] = {src, at, list, (uint32_t)cols, (uint32_t)groups, c.groups};
    c.groups += rows * groups;
    void* const dst = at;
    at += bytes(rows, cols, dtype);
    return dst;
  }
  hipError_t run(hipStream_t s) const {
    if (c.groups == 0) return hipSuccess;
    const dim3 grid((unsigned)((c.groups + 255) / 256));
    if (c.elem == 4) ffn_copy_kernel<uint32_t><<<grid, dim3(256), 0, s>>>(c);
    else ffn_copy_kernel<uint16_t><<<grid, dim3(256), 0, s>>>(c);
    return hipGetLastError();
  }
};

// Tile shape and parts of the contraction for a product of m x cols results (cols: rows of Q) and `k`, priced with what was measured, in
// us a K tile of 128 bytes of k, launches of 2 048 x 16-bit k behind each other.  `half`: half as many workgroups as there is room for, or
// fewer (the clock is higher); `full`: as many; across k on both sides the second pair.
//   128 x 128, two a compute unit   0.42, 1.06   0.62, 1.2     floats, which have these tiles alone: 1.55, 2.75
//   256 x 256                       1.05, 1.6    1.15, 1.75
//   256 x 128                       0.58, 0.8    0.72, 0.95
// A launch takes 3 us, a tile's beginning and end 5, in proportion to its rows.  A contraction in parts leaves sums in float, written and
// read once at 4 TB/s, and another launch.  6 272 x 2 048 -> 768 in bf16: 30.5, 40.9 and 26.9 us in these tiles; 8 192 x 2 048 -> 4 096:
// 113 in the second, 128 in the third.
struct FfnTileShape {
  int rows, cols, room;
  double half[2], full[2];
};
constexpr FfnTileShape kTiles[] = {{128, 128, 512, {0.42, 0.62}, {1.06, 1.2}}, {256, 256, 256, {1.05, 1.15}, {1.6, 1.75}},
                                {256, 128, 256, {0.58, 0.72}, {0.8, 0.95}}};
constexpr int kMostSplits = 32, kLeastTiles = 4;
static int64_t k_tiles_of(int64_t k, int segments, int dtype) {
  const int64_t entries = 128 / elem_bytes(dtype);
  return segments * ((k + entries - 1) / entries);
}

struct Tiling {
  int tile, splits;
  double us;
};

static Tiling pick_tiling(FfnProduct what, int64_t m, int64_t cols, int64_t k, int segments, int batch, int dtype) {
  const bool across = what == kFfnWGrad, f32 = dtype == SC_F32;
  const int64_t k_tiles = k_tiles_of(k, segments, dtype);
  Tiling best = {0, 1, 1e30};
  for (int tile = 0; tile < (f32 ? 1 : 3); ++tile) {
    const FfnTileShape& shape = kTiles[tile];
    const int64_t room = shape.room;
    const double half = f32 ? 1.55 : shape.half[across], full = f32 ? 2.75 : shape.full[across];
    const int64_t tiles = ((m + shape.rows - 1) / shape.rows) * ((cols + shape.cols - 1) / shape.cols) * batch;
    for (int splits = 1; splits <= kMostSplits; ++splits) {
      if (splits > 1 && k_tiles / splits < kLeastTiles) break;
      const int64_t count = tiles * splits, rest = count % room;
      if (splits > 1 && ((splits - 1) * tiles > (tile ? 256 : 1024) || count > 2 * room)) break;
      const double rounds = (double)(count / room), over = 2.0 * rest / room - 1.0;
      // beyond half the room, tiles of 128 share some compute units, and the slower ones count
      const double left = rest == 0 ? 0.0 : over <= 0.0 ? half : half + (full - half) * (tile == 0 ? 0.4 + 0.6 * over : over);
      const double per = (double)((k_tiles + splits - 1) / splits);
      double us = 3.0 + (rounds * full + left) * per + (rounds + (rest ? 1.0 : 0.0)) * 5.0 * std::min(1.0, (double)m / shape.rows);
      if (splits > 1) us += 4.0 + (double)splits * batch * m * cols * 8.0 / 4e6;
      if (us < best.us) best = {tile, splits, us};
    }
  }
  return best;
}

// What a workspace must hold of a result's parts, whatever the number of rows up to this one: a part has four K tiles or more, and there are
// at most kMostSplits, and at most 1 024 tiles of 128 x 128 (256 of the larger ones) besides a result that is no larger than that itself.
static size_t most_parts(int64_t m, int64_t n, int64_t k, int segments, int batch, int dtype) {
  const int64_t parts = std::min<int64_t>(kMostSplits, k_tiles_of(k, segments, dtype) / kLeastTiles);
  return parts < 2 ? 0 : up256(std::min((size_t)parts * batch * m * ((n + 3) & ~(int64_t)3) * 4, (size_t)128 << 20));
}
static size_t most_parts(const sc_ffn_desc& d, int64_t kept, bool training) {
  size_t most = std::max(most_parts(kept, d.d_hidden, d.d_in, 1, 2, d.dtype), most_parts(kept, d.d_out, d.d_hidden, 1, 1, d.dtype));
  if (training)
    most = std::max({most, most_parts(kept, d.d_hidden, d.d_out, 1, 1, d.dtype), most_parts(kept, d.d_in, d.d_hidden, 2, 1, d.dtype),
                     most_parts(d.d_hidden, d.d_in, kept, 1, 2, d.dtype), most_parts(d.d_out, d.d_hidden, kept, 1, 1, d.dtype)});
  return most;
}

// The parts added up, in order, and what the product's own epilogue would have done; 1 024 columns of a row a workgroup, blockIdx.y the result.
// Four columns a lane; rows of any length end within four (WHOLE: they do not).
template <typename T, int WHAT, bool WHOLE> __global__ __launch_bounds__(256) void ffn_finish_kernel(const FfnGemm g) {
  const int row = blockIdx.x, n = g.n, pitch = (n + 3) & ~3;
  const int64_t whole = (int64_t)g.m * n, part = (int64_t)g.m * pitch;
  auto sum = [&](int z, int i) -> v4f {
    const float* p = g.partial + z * g.splits * part + (int64_t)row * pitch + i;
    v4f v = *reinterpret_cast<const v4f*>(p);
    int s = 1;
    for (; s + 8 <= g.splits; s += 8) {      // eight on their way at once
      v4f next[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) next[u] = *reinterpret_cast<const v4f*>(p + (s + u) * part);
#pragma unroll
      for (int u = 0; u < 8; ++u) v += next[u];
    }
    for (; s + 2 <= g.splits; s += 2) {
      const v4f a = *reinterpret_cast<const v4f*>(p + s * part), b = *reinterpret_cast<const v4f*>(p + (s + 1) * part);
      v += a;
      v += b;
    }
    if (s < g.splits) v += *reinterpret_cast<const v4f*>(p + s * part);
    return v;
  };
  auto store = [&](T* c, int64_t at, int have, v4f v) {
    T out[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) out[u] = (T)v[u];
    if (WHOLE || have >= 4) {
      __builtin_memcpy(c + at, out, sizeof(out));
    } else {
#pragma unroll
      for (int u = 0; u < 3; ++u)
        if (u < have) c[at + u] = out[u];
    }
  };
  using Saved = FfnSaved<T>;
  using U = typename Saved::U;
  constexpr int PLANES = Saved::PLANES;
  U* const saved = static_cast<U*>(g.saved);
  const int i = (blockIdx.z * 256 + threadIdx.x) * 4;
  if (i < n) {
    const int64_t at = (int64_t)row * n + i, to = row * g.ldc + i;
    const int have = n - i;
    if constexpr (WHAT == kFfnUp) {
      const v4f gate = sum(0, i), up = sum(1, i);
      v4f hidden;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float a, da;
        ffn_act<T>(g.activation, gate[u], a, da);
        hidden[u] = a * up[u];
      }
      store(static_cast<T*>(g.c[0]), to, have, hidden);
      if (saved) {
        U kept[PLANES][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          U one[PLANES];
          Saved::keep(gate[u], up[u], one);
#pragma unroll
          for (int plane = 0; plane < PLANES; ++plane) kept[plane][u] = one[plane];
        }
#pragma unroll
        for (int plane = 0; plane < PLANES; ++plane) {
          if (WHOLE || have >= 4) {
            __builtin_memcpy(saved + plane * whole + at, kept[plane], sizeof(kept[plane]));
          } else {
#pragma unroll
            for (int u = 0; u < 3; ++u)
              if (u < have) saved[plane * whole + at + u] = kept[plane][u];
          }
        }
      }
    } else if constexpr (WHAT == kFfnGateGrad) {
      const v4f dh = sum(0, i);
      U kept[PLANES][4];
#pragma unroll
      for (int plane = 0; plane < PLANES; ++plane) {
        if (WHOLE || have >= 4) {
          __builtin_memcpy(kept[plane], saved + plane * whole + at, sizeof(kept[plane]));
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) kept[plane][u] = u < have ? saved[plane * whole + at + u] : U(0);
        }
      }
      v4f dg, du, hidden;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        U one[PLANES];
#pragma unroll
        for (int plane = 0; plane < PLANES; ++plane) one[plane] = kept[plane][u];
        float gate, up, a, da;
        Saved::back(one, gate, up);
        ffn_act<T>(g.activation, gate, a, da);
        dg[u] = dh[u] * up * da;
        du[u] = dh[u] * a;
        hidden[u] = a * up;
      }
      store(static_cast<T*>(g.c[0]), to, have, dg);
      store(static_cast<T*>(g.c[1]), to, have, du);
      if (g.hidden) store(static_cast<T*>(g.hidden), to, have, hidden);
    } else {
      store(static_cast<T*>(g.c[blockIdx.y]), g.c_rows ? g.c_rows[row] * g.ldc + i : to, have, sum(blockIdx.y, i));
    }
  }
  if (!WHOLE && (WHAT == kFfnUp || WHAT == kFfnGateGrad))      // zeros behind the last entry of an operand's row
    if (blockIdx.z == 0 && n + (int)threadIdx.x < g.ldc) {
      static_cast<T*>(g.c[0])[row * g.ldc + n + threadIdx.x] = T(0);
      if (WHAT == kFfnGateGrad) {
        static_cast<T*>(g.c[1])[row * g.ldc + n + threadIdx.x] = T(0);
        if (g.hidden) static_cast<T*>(g.hidden)[row * g.ldc + n + threadIdx.x] = T(0);
      }
    }
}

template <typename T, bool WHOLE> static void finish_rows(FfnProduct what, const FfnGemm& g, hipStream_t s) {
  const dim3 grid((unsigned)g.m, g.batch, (unsigned)((g.n + 1023) / 1024)), block(256);
  if (what == kFfnUp) ffn_finish_kernel<T, kFfnUp, WHOLE><<<grid, block, 0, s>>>(g);
  else if (what == kFfnGateGrad) ffn_finish_kernel<T, kFfnGateGrad, WHOLE><<<grid, block, 0, s>>>(g);
  else ffn_finish_kernel<T, kFfnDown, WHOLE><<<grid, block, 0, s>>>(g);
}
template <typename T> static void finish_type(FfnProduct what, const FfnGemm& g, bool whole, hipStream_t s) {
  if (whole) finish_rows<T, true>(what, g, s);
  else finish_rows<T, false>(what, g, s);
}
static hipError_t finish(int dtype, FfnProduct what, const FfnGemm& g, bool whole, hipStream_t s) {
  if (dtype == SC_BF16) finish_type<__bf16>(what, g, whole, s);
  else if (dtype == SC_F16) finish_type<_Float16>(what, g, whole, s);
  else finish_type<float>(what, g, whole, s);
  return hipGetLastError();
}

static hipError_t multiply(int dtype, FfnProduct what, FfnGemm& g, const Tiling& t, bool whole, float* parts, hipStream_t s) {
  g.splits = t.splits;
  g.partial = parts;
  const hipError_t e = launch(dtype, what, g, t.tile, whole, s);
  return e == hipSuccess && g.splits > 1 ? finish(dtype, what, g, whole, s) : e;
}
// a product in the tiles and parts that its sizes ask for
static hipError_t multiply(int dtype, FfnProduct what, FfnGemm& g, bool whole, float* parts, hipStream_t s) {
  return multiply(dtype, what, g, pick_tiling(what, g.m, what == kFfnUp ? 2 * (int64_t)g.n : g.n, g.k, g.segments, g.batch, dtype), whole, parts, s);
}
// kFfnUp and kFfnDown.  A few rows: the kernel for them reads all of P in every workgroup, at 4.2 TB/s in all, where the tiles' workgroups
// have eight (gated: four) times the outputs.  bf16, gated 2 048 -> 5 632 and back: 8 rows 18 us, in tiles 22; 16 rows 26 and 24; 64 rows 58
// and 30.  512 -> 1 408 and back: 64 rows 15 and 17.  Rows that are not whole groups would have to be copied for tiles, weights too.
static hipError_t multiply_forward(int dtype, FfnProduct what, FfnGemm& g, bool whole, float* parts, hipStream_t s) {
  const int64_t cols = what == kFfnUp ? 2 * (int64_t)g.n : g.n;
  const Tiling t = pick_tiling(what, g.m, cols, g.k, g.segments, g.batch, dtype);
  if (g.m > kFewRows) return multiply(dtype, what, g, t, whole, parts, s);
  if (whole) {
    const double row = (double)g.k * elem_bytes(dtype), rows = g.m <= 8 ? g.m : (g.m + 15) / 16 * 16;
    if (3.0 + cols * row / 6e6 + (g.n + 15) / 16 * rows * row / 4.2e6 > t.us) return multiply(dtype, what, g, t, whole, parts, s);
  }
  switch (dtype) {
    case SC_BF16: return ffn_few_bf16(what == kFfnUp, g, whole, s);
    case SC_F16: return ffn_few_f16(what == kFfnUp, g, whole, s);
    default: return ffn_few_f32(what == kFfnUp, g, whole, s);
  }
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
  const int dt = desc->dtype;
  const int64_t d_in = desc->d_in, d_hidden = desc->d_hidden, d_out = desc->d_out;
  const size_t hidden = sc::Copies::bytes(kept, d_hidden, dt);
  *bytes = 256 + (training ? 3 * hidden : hidden) + sc::most_parts(*desc, kept, training != 0);
  if (!sc::whole_rows(*desc)) {
    *bytes += sc::Copies::bytes(kept, d_in, dt) + 2 * sc::Copies::bytes(d_hidden, d_in, dt) + sc::Copies::bytes(d_out, d_hidden, dt);
    if (training) *bytes += sc::Copies::bytes(kept, d_out, dt);
  }
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
  if (workspace_bytes < need) return SC_ERR_WORKSPACE;
  if (sc::misaligned({x_dev, w_gate_dev, w_up_dev, w_down_dev, y_dev, saved_dev, workspace_dev})) return SC_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int eb = sc::elem_bytes(desc->dtype);
  hipError_t e = hipSuccess;
  if (y_rows == SC_ROWS_DENSE) e = sc::rows_zero_dropped(rows, (int64_t)desc->d_out * eb, y_dev, s);
  if (e != hipSuccess) return sc::failed(e);
  if (kept == 0) return SC_OK;
  const int dt = desc->dtype;
  const bool whole = sc::whole_rows(*desc), copied = !whole && kept > sc::kFewRows;
  const int64_t d_in = desc->d_in, d_hidden = desc->d_hidden, d_out = desc->d_out;
  const int64_t in_pitch = copied ? sc::pitch_of(d_in, dt) : d_in, hidden_pitch = copied ? sc::pitch_of(d_hidden, dt) : d_hidden;
  void* const hidden = workspace_dev;
  char* const w = static_cast<char*>(workspace_dev) + sc::Copies::bytes(kept, d_hidden, dt);
  float* const parts = reinterpret_cast<float*>(w);

  const int32_t* x_map = sc::map_of(rows, x_rows);
  const void *x = x_dev, *w_gate = w_gate_dev, *w_up = w_up_dev, *w_down = w_down_dev;
  if (copied) {
    sc::Copies copies(w + sc::most_parts(*desc, kept, false), dt);
    x = copies.add(x, kept, d_in, dt, x_map);
    w_gate = copies.add(w_gate, d_hidden, d_in, dt);
    w_up = copies.add(w_up, d_hidden, d_in, dt);
    w_down = copies.add(w_down, d_out, d_hidden, dt);
    x_map = nullptr;
    e = copies.run(s);
    if (e != hipSuccess) return sc::failed(e);
  }

  sc::FfnGemm up = sc::gemm_of(kept, d_hidden, d_in);
  up.p[0] = x;
  up.ldp = up.ldq = in_pitch;
  up.p_rows = x_map;
  up.q[0] = w_gate;
  up.q[1] = w_up;
  up.c[0] = hidden;
  up.ldc = hidden_pitch;
  up.saved = saved_dev;
  up.activation = desc->activation;
  e = sc::multiply_forward(dt, sc::kFfnUp, up, whole, parts, s);
  if (e != hipSuccess) return sc::failed(e);

  sc::FfnGemm down = sc::gemm_of(kept, d_out, d_hidden);
  down.p[0] = hidden;
  down.q[0] = w_down;
  down.ldp = down.ldq = hidden_pitch;
  down.c[0] = y_dev;
  down.ldc = d_out;
  down.c_rows = sc::map_of(rows, y_rows);
  e = sc::multiply_forward(dt, sc::kFfnDown, down, whole, parts, s);
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
  const int dt = desc->dtype;
  const bool whole = sc::whole_rows(*desc);
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
  const size_t hidden_bytes = sc::Copies::bytes(kept, d_hidden, dt);
  const int64_t in_pitch = sc::pitch_of(d_in, dt), hidden_pitch = sc::pitch_of(d_hidden, dt), out_pitch = sc::pitch_of(d_out, dt);
  void* const dg = w;
  void* const du = w + hidden_bytes;
  void* const hidden = w + 2 * hidden_bytes;
  float* const partial = reinterpret_cast<float*>(w + 3 * hidden_bytes);
  const int32_t *x_map = sc::map_of(rows, x_rows), *y_map = sc::map_of(rows, y_rows);
  const int32_t* const dx_map = x_map;
  const void *x = x_dev, *dy = dy_dev, *w_gate = w_gate_dev, *w_up = w_up_dev, *w_down = w_down_dev;
  if (!whole) {
    sc::Copies copies(w + 3 * hidden_bytes + sc::most_parts(*desc, kept, true), dt);
    dy = copies.add(dy, kept, d_out, dt, y_map);
    w_down = copies.add(w_down, d_out, d_hidden, dt);
    if (dx_dev) {
      w_gate = copies.add(w_gate, d_hidden, d_in, dt);
      w_up = copies.add(w_up, d_hidden, d_in, dt);
    }
    if (weights) x = copies.add(x, kept, d_in, dt, x_map);
    x_map = y_map = nullptr;
    e = copies.run(s);
    if (e != hipSuccess) return sc::failed(e);
  }

  sc::FfnGemm gate = sc::gemm_of(kept, d_hidden, d_out);       // dhidden = dY Wd, then dg and du
  gate.p[0] = dy;
  gate.ldp = out_pitch;
  gate.p_rows = y_map;
  gate.q[0] = w_down;
  gate.ldq = hidden_pitch;
  gate.saved = const_cast<void*>(saved_dev);
  gate.c[0] = dg;
  gate.c[1] = du;
  gate.hidden = weights ? hidden : nullptr;
  gate.ldc = hidden_pitch;
  gate.activation = desc->activation;
  e = sc::multiply(dt, sc::kFfnGateGrad, gate, whole, partial, s);
  if (e != hipSuccess) return sc::failed(e);

  if (dx_dev) {
    sc::FfnGemm in = sc::gemm_of(kept, d_in, d_hidden);
    in.segments = 2;
    in.p[0] = dg;
    in.p[1] = du;
    in.ldp = hidden_pitch;
    in.q[0] = w_gate;
    in.q[1] = w_up;
    in.ldq = in_pitch;
    in.c[0] = dx_dev;
    in.ldc = d_in;
    in.c_rows = dx_map;
    e = sc::multiply(dt, sc::kFfnInGrad, in, whole, partial, s);
    if (e != hipSuccess) return sc::failed(e);
  }
  if (weights) {
    sc::FfnGemm in = sc::gemm_of(d_hidden, d_in, kept);        // dWg = dg' X, dWu = du' X
    in.batch = 2;
    in.p[0] = dg;
    in.p[1] = du;
    in.ldp = hidden_pitch;
    in.q[0] = x;
    in.ldq = in_pitch;
    in.q_rows = x_map;
    in.c[0] = dw_gate_dev;
    in.c[1] = dw_up_dev;
    in.ldc = d_in;
    e = sc::multiply(dt, sc::kFfnWGrad, in, whole, partial, s);
    if (e != hipSuccess) return sc::failed(e);

    sc::FfnGemm out = sc::gemm_of(d_out, d_hidden, kept);      // dWd = dY' hidden
    out.p[0] = dy;
    out.ldp = out_pitch;
    out.p_rows = y_map;
    out.q[0] = hidden;
    out.ldq = hidden_pitch;
    out.c[0] = dw_down_dev;
    out.ldc = d_hidden;
    e = sc::multiply(dt, sc::kFfnWGrad, out, whole, partial, s);
    if (e != hipSuccess) return sc::failed(e);
  }
  return SC_OK;
}

}  // extern "C"
