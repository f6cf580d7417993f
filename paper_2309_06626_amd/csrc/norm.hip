// Norm behind a block, its gate, the residual sum and the norm before the next block, in one pass over the rows; and the gradients.
//
//   n = post(f) w_post + b_post,  x' = a x + b gate n,  h = pre(x') w_pre + b_pre
//   t = dx' + pre'(dh w_pre),  dx = a t,  q = b t,  dgate = sum q n,  r = q gate,  dw_post = sum r post(f),  db_post = sum r,
//   df = post'(r w_post),  dw_pre = sum dh pre(x'),  db_pre = sum dh
//   with post'(g) = (g - nf mean(g nf) - [layer] mean(g)) / spread,  nf the normalised row
//
// Memory bound: x, f in and x', h out are 4 accesses an element forward, x, f, dx', dh, dx, df are 6 more backward, for 14 and 30
// operations.  A row lies in the registers of one workgroup, 8 or 16 channels a lane, so that every tensor
// passes once and a layer norm's spread is summed about its mean, not from squares.  A workgroup walks over rows with the
// parameters in registers; backward their gradients too, and since its rows are consecutive, a gate's gradient is finished as its
// rows end.  What a workgroup cannot finish it leaves in float, and a second launch adds these parts in order.
// Measured, tensors from memory: 8 192 x 4 096 in bf16 forward 50 us (5.3 TB/s; a plain copy 6.3), backward of 4 096 x 4 096 50 and 5 for the
// parts (3.7 TB/s: four reductions a row), 3 137 x 410 in float (no whole groups) 8 and 15.5.
#include "../../include/sparse_block.h"
#include "mma_common.hpp"
#include "rows.hpp"

#include <algorithm>
#include <initializer_list>

namespace sc {

void note_hip_error(int32_t code);

struct NormParams {
  const void *x, *f, *gate;
  const float *w_post, *b_post, *w_pre, *b_pre;
  void *x_new, *h;
  float* stats;
  const int32_t *f_slot, *h_slot;      // null: row r is row r
  int64_t rows;
  int32_t d, post, pre;
  float eps, a, b;
  uint32_t rows_per_gate;
  // backward
  const void *dx_new, *dh;
  void *dx, *df, *dgate;
  float *dw[4];                        // w_post, b_post, w_pre, b_pre; null: not wanted
  float* parts;                        // [workgroups][4][d]
  float* gate_parts;                   // [teams][2][d]: the gate that a team's rows begin with, the one they end with
  int64_t rows_per_block;              // of a team
};

template <int CTRL, int ROWS> __device__ __forceinline__ float norm_dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float norm_wave_sum(float v) {      // in every lane
  v += norm_dpp<0x111, 0xf>(v);      // row_shr 1, 2, 4, 8: lane 15 of every 16 has their sum
  v += norm_dpp<0x112, 0xf>(v);
  v += norm_dpp<0x114, 0xf>(v);
  v += norm_dpp<0x118, 0xf>(v);
  v += norm_dpp<0x142, 0xa>(v);      // row_bcast 15 and 31: lane 63 has all
  v += norm_dpp<0x143, 0xc>(v);
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// Sums over a workgroup; two slots in turn, so that one barrier a sum is enough (who writes a slot again has passed the barrier of
// the sum between, which nobody reaches before having read this one).
template <int NT> struct NormSums {
  float (*slots)[2][8];
  int turn = 0;
  __device__ __forceinline__ void operator()(float& u, float& v) {
    u = norm_wave_sum(u);
    v = norm_wave_sum(v);
    if constexpr (NT > 64) {
      if ((threadIdx.x & 63) == 0) {
        slots[turn][0][threadIdx.x >> 6] = u;
        slots[turn][1][threadIdx.x >> 6] = v;
      }
      __syncthreads();
      u = v = 0.0f;
#pragma unroll
      for (int w = 0; w < NT / 64; ++w) {
        u += slots[turn][0][w];
        v += slots[turn][1][w];
      }
      turn ^= 1;
    }
  }
  __device__ __forceinline__ float one(float u) {
    u = norm_wave_sum(u);
    if constexpr (NT > 64) {
      if ((threadIdx.x & 63) == 0) slots[turn][0][threadIdx.x >> 6] = u;
      __syncthreads();
      u = 0.0f;
#pragma unroll
      for (int w = 0; w < NT / 64; ++w) u += slots[turn][0][w];
      turn ^= 1;
    }
    return u;
  }
};

// The channels of a lane: groups of 16 bytes, NT groups apart.  VEC: rows are whole groups, aligned; otherwise a group is accessed at
// any address, and the row's last one, if it is not whole, channel by channel.
template <typename T, int NT, int E, bool VEC> struct NormLane {
  static constexpr int V = 16 / (int)sizeof(T);
  int d, lane;
  struct Raw { T u[E]; };
  __device__ __forceinline__ int col(int e) const { return (lane + NT * (e / V)) * V + e % V; }
  __device__ __forceinline__ bool in(int e) const { return col(e) < d; }
  __device__ __forceinline__ bool whole(int q) const { return VEC ? in(q * V) : col(q * V) + V <= d; }
  __device__ __forceinline__ void fetch(const T* row, Raw& r) const {
#pragma unroll
    for (int q = 0; q < E / V; ++q) {
      if (whole(q)) {
        if constexpr (VEC) *reinterpret_cast<v4i*>(r.u + q * V) = *reinterpret_cast<const v4i*>(row + col(q * V));
        else __builtin_memcpy(r.u + q * V, row + col(q * V), 16);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r.u[q * V + i] = !VEC && in(q * V + i) ? row[col(q * V + i)] : T(0);
      }
    }
  }
  static __device__ __forceinline__ void widen(const Raw& r, float (&v)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (float)r.u[e];
  }
  __device__ __forceinline__ void load(const T* row, float (&v)[E]) const {
    Raw r;
    fetch(row, r);
    widen(r, v);
  }
  __device__ __forceinline__ void store(T* row, const float (&v)[E]) const {
#pragma unroll
    for (int q = 0; q < E / V; ++q) {
      T u[V];
#pragma unroll
      for (int i = 0; i < V; ++i) u[i] = (T)v[q * V + i];
      if (whole(q)) {
        if constexpr (VEC) {
          v4i g;
          __builtin_memcpy(&g, u, 16);
          *reinterpret_cast<v4i*>(row + col(q * V)) = g;
        } else {
          __builtin_memcpy(row + col(q * V), u, 16);
        }
      } else if constexpr (!VEC) {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (in(q * V + i)) row[col(q * V + i)] = u[i];
      }
    }
  }
  __device__ __forceinline__ void load_param(const float* p, float otherwise, float (&v)[E]) const {
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      v4f g;
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] = in(e + i) ? otherwise : 0.0f;
      if (p && (VEC ? in(e) : in(e + 3))) {
        g = *reinterpret_cast<const v4f*>(p + col(e));      // (the parameters themselves are aligned)
      } else if (!VEC && p) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (in(e + i)) g[i] = p[col(e + i)];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) v[e + i] = g[i];
    }
  }
};

// v becomes the normalised row; its mean and 1 / spread are returned
template <typename Lane, int NT, int E>
__device__ __forceinline__ void norm_row(int kind, float eps, const Lane& lane, NormSums<NT>& sums, float (&v)[E], float& mean,
                                         float& rstd) {
  mean = 0.0f;
  rstd = 1.0f;
  if (kind == SC_NORM_NONE) return;
  const float inv = 1.0f / (float)lane.d;
  if (kind == SC_NORM_LAYER) {
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += v[e];
    mean = sums.one(s) * inv;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = lane.in(e) ? v[e] - mean : 0.0f;
  }
  float q = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) q += v[e] * v[e];
  rstd = rsqrtf(sums.one(q) * inv + eps);
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] *= rstd;
}

template <typename T, int NT, int E, bool VEC> __global__ __launch_bounds__(NT) void norm_kernel(const NormParams p) {
  __shared__ float slots[2][2][8];
  NormSums<NT> sums{slots};
  using Lane = NormLane<T, NT, E, VEC>;
  const Lane lane{p.d, (int)threadIdx.x};
  float w_post[E], b_post[E], w_pre[E], b_pre[E], gate[E];
  lane.load_param(p.w_post, 1.0f, w_post);
  lane.load_param(p.b_post, 0.0f, b_post);
  lane.load_param(p.w_pre, 1.0f, w_pre);
  lane.load_param(p.b_pre, 0.0f, b_pre);
#pragma unroll
  for (int e = 0; e < E; ++e) gate[e] = 1.0f;
  uint32_t group = ~0u;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const int64_t fr = !p.f ? -1 : p.f_slot ? p.f_slot[r] : r, hr = !p.h ? -1 : p.h_slot ? p.h_slot[r] : r;
    float x[E], v[E];
    lane.load(static_cast<const T*>(p.x) + r * p.d, x);
    if (fr >= 0) lane.load(static_cast<const T*>(p.f) + fr * p.d, v);
    float mean1 = 0.0f, rstd1 = 0.0f, mean2 = 0.0f, rstd2 = 0.0f;
    if (fr >= 0 && p.gate && (uint32_t)r / p.rows_per_gate != group) {
      group = (uint32_t)r / p.rows_per_gate;
      lane.load(static_cast<const T*>(p.gate) + (int64_t)group * p.d, gate);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= p.a;
    if (fr >= 0) {
      norm_row<Lane, NT, E>(p.post, p.eps, lane, sums, v, mean1, rstd1);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] += p.b * gate[e] * (v[e] * w_post[e] + b_post[e]);
    }
    if (p.x_new) lane.store(static_cast<T*>(p.x_new) + r * p.d, x);
    if (hr >= 0) {
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = lane.in(e) ? x[e] : 0.0f;
      norm_row<Lane, NT, E>(p.pre, p.eps, lane, sums, x, mean2, rstd2);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = x[e] * w_pre[e] + b_pre[e];
      lane.store(static_cast<T*>(p.h) + hr * p.d, x);
    }
    if (p.stats && threadIdx.x == 0) *reinterpret_cast<v4f*>(p.stats + 4 * r) = v4f{mean1, rstd1, mean2, rstd2};
  }
}

// What a lane sums over the rows: in registers, or, where 16 channels a lane leave none, in LDS (its own words, no barrier).
template <int NT, int E, bool IN_LDS> struct NormAcc {
  float v[IN_LDS ? 1 : E];
  float* at;
  __device__ __forceinline__ explicit NormAcc(float* lds) : at(lds + threadIdx.x % NT) { clear(); }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if constexpr (IN_LDS) at[e * NT] = 0.0f;
      else v[e] = 0.0f;
    }
  }
  __device__ __forceinline__ void add(int e, float u) {
    if constexpr (IN_LDS) at[e * NT] += u;
    else v[e] += u;
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (IN_LDS) return at[e * NT];
    else return v[e];
  }
};
// Rows of up to 512 channels are a wavefront's: eight of them make a workgroup, each with rows of its own, and leave one part together.
template <int NT> constexpr int norm_teams() { return NT == 64 ? 8 : 1; }
template <int NT, int E> constexpr int norm_acc_bytes() { return NT * E > 4096 ? 4 * NT * E * 4 : norm_teams<NT>() > 1 ? norm_teams<NT>() * NT * E * 4 : 0; }

// PLAIN: two RMS norms and no biases, as decoders have them; the other forms keep means and gradients of biases too
template <typename T, int NT, int E, bool VEC, bool PLAIN>
__global__ __launch_bounds__(NT * norm_teams<NT>()) void norm_backward_kernel(const NormParams p) {
  __shared__ float slots[2][2][8];
  NormSums<NT> sums{slots};
  constexpr int TEAMS = norm_teams<NT>();
  using Lane = NormLane<T, NT, E, VEC>;
  Lane lane{p.d, (int)threadIdx.x % NT};
  const int64_t team = TEAMS > 1 ? (int64_t)blockIdx.x * TEAMS + __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : blockIdx.x;
  float w_post[E], b_post[E], w_pre[E], gate[E];
  auto load_params = [&]() {
    lane.load_param(p.w_post, 1.0f, w_post);
    if constexpr (!PLAIN) lane.load_param(p.b_post, 0.0f, b_post);
  };
  constexpr bool KEPT = NT * E <= 4096;      // otherwise there are no registers for the parameters: from the caches for every row
  if constexpr (KEPT) {
    load_params();
    lane.load_param(p.w_pre, 1.0f, w_pre);
  }
  extern __shared__ float acc_lds[];
  NormAcc<NT, E, false> dw_post(acc_lds);
  NormAcc<NT, E, !KEPT> dw_pre(acc_lds + NT * E), dgate(acc_lds + 3 * NT * E);
  NormAcc<NT, PLAIN ? 1 : E, !KEPT && !PLAIN> db_post(acc_lds), db_pre(acc_lds + 2 * NT * E);
#pragma unroll
  for (int e = 0; e < E; ++e) gate[e] = 1.0f;
  const float inv = 1.0f / (float)p.d;
  const int64_t r0 = team * p.rows_per_block, r1 = r0 + p.rows_per_block < p.rows ? r0 + p.rows_per_block : p.rows;
  const int64_t first_group = p.gate ? r0 / p.rows_per_gate : 0;
  int64_t group = -1, group_end = r0;
  // the gate's rows [begin, end) end, or this block's do: its gradient is complete if all of them were here
  auto leave_gate = [&]() {
    if (p.dgate) {
      const int64_t begin = group * p.rows_per_gate, end = begin + p.rows_per_gate < p.rows ? begin + p.rows_per_gate : p.rows;
      if (begin >= r0 && end <= r1) {
        float v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = dgate.get(e);
        lane.store(static_cast<T*>(p.dgate) + group * p.d, v);
      } else {
        float* part = p.gate_parts + (team * 2 + (group != first_group)) * p.d;
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (lane.in(e)) part[lane.col(e)] = dgate.get(e);
      }
    }
    dgate.clear();
  };
  // the next row is on its way while this one is summed, where there are registers for it
  typename Lane::Raw next_x, next_f, next_t, next_dh;
  int64_t next_fr = -1, next_hr = -1;
  auto fetch = [&](int64_t r) {
    next_fr = !p.f ? -1 : p.f_slot ? p.f_slot[r] : r;
    next_hr = !p.dh ? -1 : p.h_slot ? p.h_slot[r] : r;
    lane.fetch(static_cast<const T*>(p.x) + r * p.d, next_x);
    if (next_fr >= 0) lane.fetch(static_cast<const T*>(p.f) + next_fr * p.d, next_f);
    if constexpr (KEPT) {
      if (p.dx_new) lane.fetch(static_cast<const T*>(p.dx_new) + r * p.d, next_t);
      if (next_hr >= 0) lane.fetch(static_cast<const T*>(p.dh) + next_hr * p.d, next_dh);
    }
  };
  if (KEPT && r0 < r1) fetch(r0);
  for (int64_t r = r0; r < r1; ++r) {
    float x[E], f[E], t[E], dh[E];
    if constexpr (!KEPT) {
      __builtin_amdgcn_sched_barrier(0);      // (nothing of this row before the last one's end, and no addresses kept: registers)
      asm volatile("" : "+v"(lane.lane));
      fetch(r);
    }
    const int64_t fr = next_fr, hr = next_hr;
    Lane::widen(next_x, x);
    if (fr >= 0) Lane::widen(next_f, f);
    if (KEPT && p.dx_new) Lane::widen(next_t, t);
    if (KEPT && hr >= 0) Lane::widen(next_dh, dh);
    if (KEPT && r + 1 < r1) fetch(r + 1);
    const v4f st = *reinterpret_cast<const v4f*>(p.stats + 4 * r);
    if constexpr (!KEPT) load_params();
    if (p.gate && r == group_end) {
      if (group >= 0) leave_gate();
      group = group < 0 ? first_group : group + 1;
      group_end = (group + 1) * p.rows_per_gate;
      lane.load(static_cast<const T*>(p.gate) + group * p.d, gate);
    }
    if (!p.dx_new) {
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] = 0.0f;
    }
    if (fr >= 0 && (PLAIN || p.post != SC_NORM_NONE)) {
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = (PLAIN ? f[e] : f[e] - st[0]) * st[1];
    }
    if (hr >= 0) {
      // x becomes the normalised row of x'
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x[e] *= p.a;
        if (fr >= 0) x[e] += p.b * gate[e] * (PLAIN ? f[e] * w_post[e] : f[e] * w_post[e] + b_post[e]);
        if constexpr (PLAIN) x[e] *= st[3];
        else if (p.pre != SC_NORM_NONE) x[e] = (x[e] - st[2]) * st[3];
      }
      if constexpr (!KEPT) {
        __builtin_amdgcn_sched_barrier(0);
        lane.load(static_cast<const T*>(p.dh) + hr * p.d, dh);
        lane.load_param(p.w_pre, 1.0f, w_pre);
      }
      float s = 0.0f, u = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        dw_pre.add(e, dh[e] * x[e]);      // (beyond the row's end dh and the weights are 0, and so is what follows)
        if constexpr (!PLAIN) db_pre.add(e, dh[e]);
        dh[e] *= w_pre[e];
        s += dh[e] * x[e];
        if constexpr (!PLAIN) u += dh[e];
      }
      if (PLAIN || p.pre != SC_NORM_NONE) {
        if constexpr (PLAIN) s = sums.one(s);
        else sums(s, u);
        s *= inv;
        u = !PLAIN && p.pre == SC_NORM_LAYER ? u * inv : 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) dh[e] = st[3] * (PLAIN ? dh[e] - x[e] * s : dh[e] - x[e] * s - u);
      }
    }
    if (!KEPT && p.dx_new) {
      __builtin_amdgcn_sched_barrier(0);
      lane.load(static_cast<const T*>(p.dx_new) + r * p.d, t);
    }
    if (hr >= 0) {
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] += dh[e];
    }
    if (p.dx) {
      float dx[E];
#pragma unroll
      for (int e = 0; e < E; ++e) dx[e] = p.a * t[e];
      lane.store(static_cast<T*>(p.dx) + r * p.d, dx);
    }
    if constexpr (!KEPT) {
      __builtin_amdgcn_sched_barrier(0);
      load_params();
    }
    if (fr >= 0) {
      float s = 0.0f, u = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float q = p.b * t[e], n = PLAIN ? f[e] * w_post[e] : f[e] * w_post[e] + b_post[e];
        dgate.add(e, q * n);
        const float g = q * gate[e];
        dw_post.add(e, g * f[e]);
        if constexpr (!PLAIN) db_post.add(e, g);
        t[e] = g * w_post[e];
        s += t[e] * f[e];
        if constexpr (!PLAIN) u += t[e];
      }
      if (p.df) {
        if (PLAIN || p.post != SC_NORM_NONE) {
          if constexpr (PLAIN) s = sums.one(s);
          else sums(s, u);
          s *= inv;
          u = !PLAIN && p.post == SC_NORM_LAYER ? u * inv : 0.0f;
#pragma unroll
          for (int e = 0; e < E; ++e) t[e] = st[1] * (PLAIN ? t[e] - f[e] * s : t[e] - f[e] * s - u);
        }
        lane.store(static_cast<T*>(p.df) + fr * p.d, t);
      }
    }
  }
  if (group >= 0) leave_gate();
  auto leave = [&](int k, const auto& acc) {
    if (!p.dw[k]) return;
    float* part = p.parts + ((int64_t)blockIdx.x * 4 + k) * p.d;
    if constexpr (TEAMS == 1) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (lane.in(e)) part[lane.col(e)] = acc.get(e);
    } else {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) acc_lds[threadIdx.x / NT * (NT * E) + lane.col(e)] = acc.get(e);
      __syncthreads();
      for (int c = threadIdx.x; c < p.d; c += TEAMS * NT) {
        float v = 0.0f;
#pragma unroll
        for (int u = 0; u < TEAMS; ++u) v += acc_lds[u * (NT * E) + c];
        part[c] = v;
      }
    }
  };
  leave(0, dw_post);
  leave(2, dw_pre);
  if constexpr (!PLAIN) {
    leave(1, db_post);
    leave(3, db_pre);
  }
}

// The parts added up, in order, 32 columns a workgroup and eight lanes of parts a column: the parameters wanted, then the gates (whose rows
// lie in more than one team's stretch of p.rows_per_block; in all of these but the first the gate is the one that the stretch begins with).
// Gates of fewer rows than a stretch cross one border between stretches or none: a workgroup has 256 columns of a border then, since there may
// be a gate for every row or two and there are no more borders than teams (4 096 x 4 096 in bf16, two rows a gate, forward and backward: 85 us;
// 234 with workgroups for every gate, which beyond 2^32 lanes were no launch any more).
template <typename T> __global__ __launch_bounds__(256) void norm_finish_kernel(const NormParams p, int blocks, int params) {
  __shared__ float s[8][32];
  const int col_blocks = (p.d + 31) / 32;
  if (p.rows_per_gate < p.rows_per_block && (int)blockIdx.x >= params * col_blocks) {
    const int wide = (p.d + 255) / 256, at = blockIdx.x - params * col_blocks, border = at / wide;
    const int c = (at - border * wide) * 256 + threadIdx.x;
    const int64_t row = (border + 1) * p.rows_per_block, group = row / p.rows_per_gate;
    if (group * p.rows_per_gate == row || c >= p.d) return;      // (a gate begins there)
    const float* part = p.gate_parts + c;
    static_cast<T*>(p.dgate)[group * p.d + c] = (T)(part[((int64_t)border * 2 + 1) * p.d] + part[((int64_t)border + 1) * 2 * p.d]);
    return;
  }
  const int what = blockIdx.x / col_blocks, c = (blockIdx.x - what * col_blocks) * 32 + (threadIdx.x & 31), share = threadIdx.x >> 5;
  float v = 0.0f;
  float* out = nullptr;
  const int64_t group = what - params;
  if (what < params) {
    int k = 0;      // the what-th parameter that is wanted
    for (int seen = 0; k < 4; ++k)
      if (p.dw[k] && seen++ == what) break;
    out = p.dw[k];
    const int per = (blocks + 7) / 8, lo = share * per, hi = lo + per < blocks ? lo + per : blocks;
    if (c < p.d) {
      const float* part = p.parts + (int64_t)k * p.d + c;
#pragma unroll 8
      for (int b = lo; b < hi; ++b) v += part[(int64_t)b * 4 * p.d];
    }
  } else {
    const int64_t begin = group * p.rows_per_gate, end = begin + p.rows_per_gate < p.rows ? begin + p.rows_per_gate : p.rows;
    const int64_t lo = begin / p.rows_per_block, hi = (end - 1) / p.rows_per_block + 1;
    if (lo + 1 == hi) return;      // finished there
    const int64_t per = (hi - lo + 7) / 8, b0 = lo + share * per, b1 = b0 + per < hi ? b0 + per : hi;
    if (c < p.d) {
      const float* part = p.gate_parts + c;
      int64_t b = b0;
      if (b == lo && b < b1) v = part[(b++ * 2 + (begin > lo * p.rows_per_block)) * p.d];
#pragma unroll 8
      for (; b < b1; ++b) v += part[b * 2 * p.d];
    }
  }
  s[share][threadIdx.x & 31] = v;
  __syncthreads();
  if (share == 0 && c < p.d) {
#pragma unroll
    for (int i = 1; i < 8; ++i) v += s[i][threadIdx.x];
    if (out) out[c] = v;
    else static_cast<T*>(p.dgate)[group * p.d + c] = (T)v;
  }
}

constexpr int32_t kNormMost = 8192;      // channels: 512 lanes of 16

// ---- host ---------------------------------------------------------------------------------------------------------------------
static size_t norm_up(size_t n) { return (n + 255) & ~(size_t)255; }

// Teams of the backward pass: every workgroup leaves parts as large as a few rows, so there is one of eight wavefronts a compute unit, or
// as many lanes in smaller ones.
static int norm_team_size(int d) { return d <= 512 ? 64 : d <= 1024 ? 128 : d <= 2048 ? 256 : 512; }
static int64_t norm_most_teams(int d) { return 256 * 512 / norm_team_size(d); }
static int norm_teams_together(int d) { return d <= 512 ? 8 : 1; }
static int64_t norm_rows_per_team(int64_t rows, int d) {
  const int64_t most = norm_most_teams(d);
  return rows > 0 ? (rows + most - 1) / most : 1;
}
static int64_t norm_team_count(int64_t rows, int d) {
  const int64_t per = norm_rows_per_team(rows, d);
  return (rows + per - 1) / per;
}
static int64_t norm_block_count(int64_t rows, int d) {
  return (norm_team_count(rows, d) + norm_teams_together(d) - 1) / norm_teams_together(d);
}

template <typename T, int NT, int E, bool VEC> static hipError_t norm_launch(const NormParams& p, bool backward, hipStream_t s) {
  if (backward) {
    constexpr int lds = norm_acc_bytes<NT, E>();
    const bool plain = p.post == SC_NORM_RMS && p.pre == SC_NORM_RMS && !p.b_post && !p.dw[1] && !p.dw[3];
    auto kernel = plain ? norm_backward_kernel<T, NT, E, VEC, true> : norm_backward_kernel<T, NT, E, VEC, false>;
    if constexpr (lds > 65536) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (e != hipSuccess) return e;
    }
    kernel<<<dim3((unsigned)norm_block_count(p.rows, p.d)), dim3(NT * norm_teams<NT>()), lds, s>>>(p);
  } else {
    // rows that a workgroup takes after one another spare it the parameters; short rows gain more from more workgroups
    // (12 544 x 768 in f16: 2 048 workgroups 19.1 us, 8 192 17.9; 8 192 x 4 096 in bf16: 512 51.5, 2 048 53.2)
    const int64_t most = NT <= 128 ? 8192 : 262144 / NT;
    norm_kernel<T, NT, E, VEC><<<dim3((unsigned)(p.rows < most ? p.rows : most)), dim3(NT), 0, s>>>(p);
  }
  return hipGetLastError();
}

template <typename T, bool VEC> static hipError_t norm_launch_width(const NormParams& p, bool backward, hipStream_t s) {
  if (p.d <= 512) return norm_launch<T, 64, 8, VEC>(p, backward, s);
  if (p.d <= 1024) return norm_launch<T, 128, 8, VEC>(p, backward, s);
  if (p.d <= 2048) return norm_launch<T, 256, 8, VEC>(p, backward, s);
  if (p.d <= 4096) return norm_launch<T, 512, 8, VEC>(p, backward, s);
  return norm_launch<T, 512, 16, VEC>(p, backward, s);
}

template <typename T> static hipError_t norm_launch_type(const NormParams& p, bool backward, hipStream_t s) {
  return (size_t)p.d * sizeof(T) % 16 == 0 ? norm_launch_width<T, true>(p, backward, s) : norm_launch_width<T, false>(p, backward, s);
}

static hipError_t norm_dispatch(int dtype, const NormParams& p, bool backward, hipStream_t s) {
  if (dtype == SC_BF16) return norm_launch_type<__bf16>(p, backward, s);
  if (dtype == SC_F16) return norm_launch_type<_Float16>(p, backward, s);
  return norm_launch_type<float>(p, backward, s);
}

static sc_status check_norm(const sc_norm_desc* d, int64_t rows) {
  if (!d) return SC_ERR_NULL;
  if (d->dtype != SC_F32 && d->dtype != SC_F16 && d->dtype != SC_BF16) return SC_ERR_UNSUPPORTED;
  for (int k : {d->post, d->pre})
    if (k < SC_NORM_NONE || k > SC_NORM_LAYER) return SC_ERR_UNSUPPORTED;
  if (d->d < 1 || d->d > kNormMost || rows < 0 || rows > 0x7fffffff || d->rows_per_gate < 0 || !(d->eps >= 0.0f)) return SC_ERR_BAD_SHAPE;
  return SC_OK;
}

static bool norm_misaligned(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if ((uintptr_t)p & 15) return true;
  return false;
}

static NormParams norm_params(const sc_norm_desc* d, int64_t rows) {
  NormParams p = {};
  p.rows = rows;
  p.d = d->d;
  p.post = d->post;
  p.pre = d->pre;
  p.eps = d->eps;
  p.a = d->residual_scale;
  p.b = d->branch_scale;
  p.rows_per_gate = d->rows_per_gate ? d->rows_per_gate : rows > 0 ? (uint32_t)rows : 1;
  return p;
}

// a matrix of kept rows: nothing where none is kept
template <typename P> static P* norm_kept(P* matrix, const sc_rows* set) { return set && set->kept == 0 ? nullptr : matrix; }
// null where every row is kept
static const int32_t* norm_slots(const sc_rows* set) { return set && set->kept != set->rows ? set->slot : nullptr; }

}  // namespace sc

extern "C" {

sc_status sparse_norm_run(const sc_norm_desc* desc, int64_t rows, const void* x_dev, const void* f_dev, const sc_rows* f_rows,
                          const void* gate_dev, const float* w_post_dev, const float* b_post_dev, const float* w_pre_dev,
                          const float* b_pre_dev, void* x_new_dev, void* h_dev, const sc_rows* h_rows, float* stats_dev,
                          void* hip_stream) {
  const sc_status st = sc::check_norm(desc, rows);
  if (st != SC_OK) return st;
  if ((f_rows && f_rows->rows != rows) || (h_rows && h_rows->rows != rows)) return SC_ERR_BAD_SHAPE;
  if (rows > 0 && (!x_dev || (!x_new_dev && !h_dev && !(h_rows && h_rows->kept == 0)))) return SC_ERR_NULL;
  if (sc::norm_misaligned({x_dev, f_dev, gate_dev, w_post_dev, b_post_dev, w_pre_dev, b_pre_dev, x_new_dev, h_dev, stats_dev}))
    return SC_ERR_ALIGN;
  if (rows == 0) return SC_OK;
  sc::NormParams p = sc::norm_params(desc, rows);
  p.x = x_dev;
  p.f = sc::norm_kept(f_dev, f_rows);
  p.gate = gate_dev;
  p.w_post = w_post_dev;
  p.b_post = b_post_dev;
  p.w_pre = w_pre_dev;
  p.b_pre = b_pre_dev;
  p.x_new = x_new_dev;
  p.h = sc::norm_kept(h_dev, h_rows);
  p.stats = stats_dev;
  p.f_slot = sc::norm_slots(f_rows);
  p.h_slot = sc::norm_slots(h_rows);
  const hipError_t e = sc::norm_dispatch(desc->dtype, p, false, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) { sc::note_hip_error((int32_t)e); return SC_ERR_HIP; }
  return SC_OK;
}

sc_status sparse_norm_workspace_bytes(const sc_norm_desc* desc, int64_t rows, size_t* bytes) {
  if (!bytes) return SC_ERR_NULL;
  *bytes = 0;
  const sc_status st = sc::check_norm(desc, rows);
  if (st != SC_OK) return st;
  // (as many as there can be for up to this many rows)
  const int64_t teams = std::min(rows, sc::norm_most_teams(desc->d)), together = sc::norm_teams_together(desc->d);
  *bytes = 256 + sc::norm_up((size_t)((teams + together - 1) / together) * 4 * desc->d * 4) + sc::norm_up((size_t)teams * 2 * desc->d * 4);
  return SC_OK;
}

sc_status sparse_norm_backward(const sc_norm_desc* desc, int64_t rows, const void* x_dev, const void* f_dev, const sc_rows* f_rows,
                               const void* gate_dev, const float* w_post_dev, const float* b_post_dev, const float* w_pre_dev,
                               const float* stats_dev, const void* dx_new_dev, const void* dh_dev, const sc_rows* h_rows,
                               void* dx_dev, void* df_dev, void* dgate_dev, float* dw_post_dev, float* db_post_dev,
                               float* dw_pre_dev, float* db_pre_dev, void* workspace_dev, size_t workspace_bytes,
                               void* hip_stream) {
  const sc_status st = sc::check_norm(desc, rows);
  if (st != SC_OK) return st;
  if ((f_rows && f_rows->rows != rows) || (h_rows && h_rows->rows != rows)) return SC_ERR_BAD_SHAPE;
  // (a matrix of no rows may have no address)
  if ((rows > 0 && (!x_dev || !stats_dev || (!dx_new_dev && !dh_dev && !(h_rows && h_rows->kept == 0)))) || !workspace_dev) return SC_ERR_NULL;
  if (rows > 0 && !f_dev && (!f_rows || f_rows->kept > 0) && (df_dev || dgate_dev || dw_post_dev || db_post_dev)) return SC_ERR_NULL;
  if (dgate_dev && !gate_dev) return SC_ERR_NULL;
  if (rows > 0 && !dh_dev && (!h_rows || h_rows->kept > 0) && (dw_pre_dev || db_pre_dev)) return SC_ERR_NULL;
  size_t need = 0;
  sparse_norm_workspace_bytes(desc, rows, &need);
  if (workspace_bytes < need) return SC_ERR_WORKSPACE;
  if (sc::norm_misaligned({x_dev, f_dev, gate_dev, w_post_dev, b_post_dev, w_pre_dev, stats_dev, dx_new_dev, dh_dev, dx_dev, df_dev,
                           dgate_dev, dw_post_dev, db_post_dev, dw_pre_dev, db_pre_dev, workspace_dev}))
    return SC_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  sc::NormParams p = sc::norm_params(desc, rows);
  p.x = x_dev;
  p.f = sc::norm_kept(f_dev, f_rows);
  p.gate = gate_dev;
  p.w_post = w_post_dev;
  p.b_post = b_post_dev;
  p.w_pre = w_pre_dev;
  p.stats = const_cast<float*>(stats_dev);
  p.f_slot = sc::norm_slots(f_rows);
  p.h_slot = sc::norm_slots(h_rows);
  p.dx_new = dx_new_dev;
  p.dh = sc::norm_kept(dh_dev, h_rows);
  p.dx = dx_dev;
  p.df = df_dev;
  p.dgate = dgate_dev;
  float* const grads[4] = {dw_post_dev, db_post_dev, dw_pre_dev, db_pre_dev};
  int params = 0;
  for (int k = 0; k < 4; ++k) {
    p.dw[k] = grads[k];
    params += grads[k] != nullptr;
  }
  p.rows_per_block = sc::norm_rows_per_team(rows, desc->d);
  const int64_t blocks = sc::norm_block_count(rows, desc->d);
  p.parts = static_cast<float*>(workspace_dev);
  p.gate_parts = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + sc::norm_up((size_t)blocks * 4 * desc->d * 4));
  hipError_t e = hipSuccess;
  if (rows > 0) e = sc::norm_dispatch(desc->dtype, p, true, s);
  const int64_t teams = sc::norm_team_count(rows, desc->d), col_blocks = (desc->d + 31) / 32;
  int64_t units = params * col_blocks;
  if (rows > 0 && dgate_dev && teams > 1) {      // gates that no team finished: no more than there are borders between teams
    if (p.rows_per_gate >= p.rows_per_block) units += (rows + p.rows_per_gate - 1) / p.rows_per_gate * col_blocks;
    else if (p.rows_per_block % p.rows_per_gate) units += (teams - 1) * ((desc->d + 255) / 256);
  }
  if (e == hipSuccess && units > 0) {
    const dim3 grid((unsigned)units);
    if (desc->dtype == SC_BF16) sc::norm_finish_kernel<__bf16><<<grid, dim3(256), 0, s>>>(p, (int)blocks, params);
    else if (desc->dtype == SC_F16) sc::norm_finish_kernel<_Float16><<<grid, dim3(256), 0, s>>>(p, (int)blocks, params);
    else sc::norm_finish_kernel<float><<<grid, dim3(256), 0, s>>>(p, (int)blocks, params);
    e = hipGetLastError();
  }
  if (e != hipSuccess) { sc::note_hip_error((int32_t)e); return SC_ERR_HIP; }
  return SC_OK;
}

}  // extern "C"
