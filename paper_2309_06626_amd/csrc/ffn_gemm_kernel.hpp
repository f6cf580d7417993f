// Products of the gated feed-forward block: C[i][j] = sum_k P[i][k] Q[j][k] in tiles of BM x BN on the matrix cores, with the
// block's activation, gating and row maps in the loads and the epilogue.
#pragma once
#include "ffn_act.hpp"
#include "ffn_params.hpp"
#include "mma_common.hpp"

namespace sc {

// ---- LDS tiles ------------------------------------------------------------------------------------------------------------------
// 128 bytes of k a row of an operand along k (64 entries of 16 bits, 32 floats); an operand across k has as many rows of k.
// A 16-byte group lies at its index XOR a key of its row, so that the lanes that read together touch every bank once.
template <int EB> struct FfnTile {
  static constexpr int BK = 128 / EB, V = 16 / EB, STEPS = 4, KSTEP = BK / STEPS;
  // sixteen lanes read at once: two rows of one group side by side in the 256 bytes of the banks, eight such pairs; the rows are
  // consecutive (P) or those of ffn_q_order, 0 .. 7 and 16 .. 23
  static __device__ __forceinline__ int key_along(int row) { return ((row >> 1) & 3) | ((((row >> 3) ^ (row >> 4)) & 1) << 2); }
  static __device__ __forceinline__ int key_across(int k) {
    if constexpr (EB == 2) return ((k & 3) << 2) | ((k >> 1) & 1);
    return ((k >> 2) & 1) << 3;
  }
};

// A 32 x 32 block of results leaves 16 registers a lane: with the Q rows of a block read in this order, they are 16 consecutive
// columns of the lane's row.
__device__ __forceinline__ int ffn_q_order(int r) { return ((r >> 2) & 1) * 16 + (r >> 3) * 4 + (r & 3); }

constexpr int kFfnList = 4096;      // rows of the contraction whose list entries lie in LDS
static __device__ __align__(16) v4i ffn_zeros = {0, 0, 0, 0};      // what is read beyond an operand's end

// 16 bytes a lane from memory into LDS at base + 16 lane.  Written out, because the compiler would let every later LDS read wait
// for all transfers in flight; their arrival is waited for at the barriers below.
__device__ __forceinline__ void ffn_dma16(const void* src, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_base), "v"(src));
}

template <int I, int N, class Fn> __device__ __forceinline__ void ffn_for(Fn&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    ffn_for<I + 1, N>(f);
  }
}

template <int DT, bool P_ALONG, bool Q_ALONG, int WHAT, int BM, int BN, int WAVES_M, int WAVES_N, bool ALIGNED>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) void ffn_gemm_kernel(const FfnGemm p) {
  using E = Elem<DT>;
  using T = typename E::T;
  constexpr int EB = sizeof(T);
  using L = FfnTile<EB>;
  constexpr int V = L::V, BK = L::BK;
  constexpr int W = WAVES_M * WAVES_N, NT = 64 * W;
  constexpr int MI = BM / WAVES_M / 32, NI = BN / WAVES_N / 32;
  constexpr int JP = BM * 8 / NT, JQ = BN * 8 / NT;            // transfers a lane and K tile
  constexpr int P_BYTES = BM * 128, STAGE = (BM + BN) * 128;
  constexpr bool GATED = WHAT == kFfnUp;
  constexpr int HALF = GATED ? NI / 2 : NI;                    // blocks of columns that a wavefront leaves
  constexpr int COLS = GATED ? BN / 2 : BN;                    // result columns of a tile
  extern __shared__ __align__(16) unsigned char smem[];

  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave / WAVES_N, wn = wave % WAVES_N;
  const int l32 = lane & 31, h = lane >> 5;

  // consecutive workgroups go round the eight dies: renumbered so that a die has neighbouring tiles, `group` tiles high
  const int tiles = p.m_tiles * p.n_tiles, total = tiles * p.batch * p.splits;
  const int per_xcd = (total + 7) >> 3;
  int at = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per_xcd || at >= total) return;
  const int part = at / tiles;
  at -= part * tiles;
  const int z = part / p.splits, split = part - z * p.splits;
  const int band = at / (p.group * p.n_tiles), in_band = at - band * p.group * p.n_tiles;
  const int high = min(p.group, p.m_tiles - band * p.group);
  const int m0 = (band * p.group + in_band % high) * BM, n0 = (in_band / high) * COLS;

  // K tiles of this workgroup: every segment is a whole number of tiles, the last one padded with zeros
  const int n_last = p.n - 1;
  const bool q_listed = p.q_rows != nullptr;
  const int seg_tiles = (p.k + BK - 1) / BK, all_tiles = seg_tiles * p.segments;
  const int kt_lo = (int)((int64_t)all_tiles * split / p.splits), kt_hi = (int)((int64_t)all_tiles * (split + 1) / p.splits);

  // ---- loads ----
  // slot s of an operand's tile (16 bytes): along k, row s / 8, group s % 8; across k, row s / CPR of k, group s % CPR
  constexpr int P_CPR = P_ALONG ? 8 : BM / V, Q_CPR = Q_ALONG ? 8 : BN / V;
  const int p_row = wave * (64 / P_CPR) + lane / P_CPR, q_row = wave * (64 / Q_CPR) + lane / Q_CPR;      // of transfer 0
  constexpr int P_NEXT = W * (64 / P_CPR), Q_NEXT = W * (64 / Q_CPR);                                    // rows from transfer to transfer
  // k (along) or result row / column (across) of the lane's group; the same for all its transfers, whose rows have one key
  const int p_at = P_ALONG ? ((lane & 7) ^ L::key_along(p_row)) * V : m0 + ((lane % P_CPR) ^ L::key_across(p_row)) * V;
  const int q_at = Q_ALONG ? ((lane & 7) ^ L::key_along(q_row)) * V : n0 + ((lane % Q_CPR) ^ L::key_across(q_row)) * V;
  int64_t pp[P_ALONG ? JP : 1], qq_at[Q_ALONG ? JQ : 1];      // from the start of the operand
  const T* qq[Q_ALONG && GATED ? JQ : 1];                      // two matrices: addresses
  // held in scalar registers: a load of a kernel argument between the products would have to wait for the operands on their way
  const T *p0 = static_cast<const T*>(p.p[P_ALONG ? 0 : z]), *p1 = static_cast<const T*>(p.p[p.segments > 1]);
  const T *q0 = static_cast<const T*>(p.q[0]), *q1 = static_cast<const T*>(p.q[p.segments > 1]);
  int64_t ldp = p.ldp, ldq = p.ldq;
  int k_end = p.k;
  const void* zeros = &ffn_zeros;
  asm volatile("" : "+s"(p0), "+s"(p1), "+s"(q0), "+s"(q1), "+s"(ldp), "+s"(ldq), "+s"(k_end), "+s"(zeros));
  if constexpr (P_ALONG) {
#pragma unroll
    for (int j = 0; j < JP; ++j) {
      const int i = min(m0 + p_row + j * P_NEXT, p.m - 1);      // rows beyond the end: results that are not stored
      pp[j] = (p.p_rows ? (int64_t)p.p_rows[i] : i) * ldp + p_at;
    }
  }
  if constexpr (Q_ALONG) {
#pragma unroll
    for (int j = 0; j < JQ; ++j) {
      const int r = q_row + j * Q_NEXT, up = GATED && r >= COLS;
      const int c = min(n0 + (up ? r - COLS : r), n_last);
      qq_at[j] = c * ldq + q_at;
      if constexpr (GATED) qq[j] = static_cast<const T*>(p.q[up]) + qq_at[j];
    }
  }
  // rows of the contraction that stand for others: a stretch of the list at a time in LDS (a look-up in memory would have to wait
  // for the transfers before it)
  constexpr bool LISTED = WHAT == kFfnWGrad;
  int32_t* const s_list = reinterpret_cast<int32_t*>(smem + (ALIGNED ? 2 : 1) * STAGE);
  const int32_t* const list = LISTED ? (p.p_rows ? p.p_rows : p.q_rows) : nullptr;
  int list_base = 0;
  auto stretch = [&](int kt) {      // called by all
    list_base = kt * BK;
    for (int i = t; i < kFfnList && list_base + i < p.k; i += NT) s_list[i] = list[list_base + i];
  };
  auto p_k = [&](int k) -> int64_t { return LISTED && p.p_rows ? s_list[k - list_base] : k; };
  auto q_k = [&](int k) -> int64_t { return LISTED && q_listed ? s_list[k - list_base] : k; };

  const unsigned lds0 = (unsigned)(unsigned long long)(__attribute__((address_space(3))) unsigned char*)smem;
  // columns beyond the end across k: any that exist
  const int p_in = min(p_at, p.m - V), q_in = min(q_at, p.n - V);
  int32_t listed_row[P_ALONG ? JQ : (JP > JQ ? JP : JQ)];      // of the tile asked for next
  auto look_up = [&](int kt) {
    if constexpr (LISTED) {
      if (!list) return;
      const int first = kt * BK + (q_listed ? q_row : p_row), next = q_listed ? Q_NEXT : P_NEXT;
#pragma unroll
      for (int j = 0; j < (JP > JQ ? JP : JQ); ++j) listed_row[j] = s_list[min(first + j * next, p.k - 1) - list_base];
    }
  };
  // What the transfers of a K tile share, worked out once: whole groups go straight into LDS, zeros beyond the end of k.
  struct Ask { const T *p, *q; int k0; unsigned to; };
  auto prepare = [&](int kt, int stage) -> Ask {
    const int seg = kt >= seg_tiles, k0 = (kt - seg * seg_tiles) * BK;
    Ask a;
    a.k0 = k0;
    a.to = lds0 + stage * STAGE + wave * 1024;
    a.p = P_ALONG ? (seg ? p1 : p0) + k0 : p0;
    a.q = (seg ? q1 : q0) + (Q_ALONG ? k0 : 0);
    return a;
  };
  auto request_one = [&](const Ask& a, auto which) {
    constexpr int j = decltype(which)::value;
    const T* src;
    bool in;
    if constexpr (j < JP) {
      if constexpr (P_ALONG) {
        src = a.p + pp[j];
        in = a.k0 + p_at < k_end;
      } else {
        const int k = a.k0 + p_row + j * P_NEXT;
        in = k < k_end;
        src = a.p + p_in + (LISTED && list && !q_listed ? listed_row[j] : in ? k : 0) * ldp;
      }
      ffn_dma16(in ? (const void*)src : zeros, a.to + j * NT * 16);
    } else {
      constexpr int i = j - JP;
      if constexpr (Q_ALONG) {
        if constexpr (GATED) src = qq[i] + a.k0;
        else src = a.q + qq_at[i];
        in = a.k0 + q_at < k_end;
      } else {
        const int k = a.k0 + q_row + i * Q_NEXT;
        in = k < k_end;
        src = a.q + q_in + (LISTED && q_listed ? listed_row[i] : in ? k : 0) * ldq;
      }
      ffn_dma16(in ? (const void*)src : zeros, a.to + P_BYTES + i * NT * 16);
    }
  };
  // the source of transfer j of K tile kt, and how many of its entries there are (rows of any length)
  auto p_src = [&](int kt, int j, int& have) -> const T* {
    const int seg = kt >= seg_tiles, k0 = (kt - seg * seg_tiles) * BK;
    if constexpr (P_ALONG) {
      have = min(V, p.k - (k0 + p_at));
      return (seg ? p1 : p0) + pp[j] + k0;
    } else {
      const int k = k0 + p_row + j * P_NEXT;
      have = k < p.k ? min(V, p.m - p_at) : 0;
      return p0 + (have > 0 ? p_k(k) * ldp + p_at : 0);
    }
  };
  auto q_src = [&](int kt, int j, int& have) -> const T* {
    const int seg = kt >= seg_tiles, k0 = (kt - seg * seg_tiles) * BK;
    if constexpr (Q_ALONG) {
      have = min(V, p.k - (k0 + q_at));
      if constexpr (GATED) return qq[j] + k0;
      else return q0 + qq_at[j] + k0;
    } else {
      const int k = k0 + q_row + j * Q_NEXT;
      have = k < p.k ? min(V, p.n - q_at) : 0;
      return (seg ? q1 : q0) + (have > 0 ? q_k(k) * ldq + q_at : 0);
    }
  };
  v4i held[JP + JQ];                                           // rows of any length: through registers
  auto load_group = [=](const T* s, int have) -> v4i {
    if (have >= V) {
      v4i g;
      __builtin_memcpy(&g, s, 16);
      return g;
    }
    T e[V];
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = i < have ? s[i] : T(0);
    v4i g;
    __builtin_memcpy(&g, e, 16);
    return g;
  };
  auto hold = [&](int kt) {
#pragma unroll
    for (int j = 0; j < JP; ++j) {
      int have;
      const T* s = p_src(kt, j, have);
      held[j] = load_group(s, have);
    }
#pragma unroll
    for (int j = 0; j < JQ; ++j) {
      int have;
      const T* s = q_src(kt, j, have);
      held[JP + j] = load_group(s, have);
    }
  };
  auto put = [&]() {
#pragma unroll
    for (int j = 0; j < JP; ++j) *reinterpret_cast<v4i*>(smem + (j * NT + t) * 16) = held[j];
#pragma unroll
    for (int j = 0; j < JQ; ++j) *reinterpret_cast<v4i*>(smem + P_BYTES + (j * NT + t) * 16) = held[JP + j];
  };

  // ---- fragments ----
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  // 32 rows r0 .. r0 + 31 of an operand's tile (of BR rows), KSTEP entries of k
  auto fragment = [&](auto along, auto is_q, const unsigned char* tile, auto br, int r0, int ks) -> v4i {
    constexpr int BR = decltype(br)::value;
    if constexpr (decltype(along)::value) {
      const int r = decltype(is_q)::value ? ffn_q_order(l32) : l32;
      return *reinterpret_cast<const v4i*>(tile + (r0 + r) * 128 + (((2 * ks + h) ^ L::key_along(r)) << 4));
    } else if constexpr (EB == 2) {
      // within 16 lanes the transposing read gives lane j element t of source lane 4 t + j / 4, entry j % 4: source lane s
      // points at row s / 4 of k, columns of the four lanes from 4 (s % 4) on
      const int l16 = lane & 15, k = ks * L::KSTEP + 8 * h + (l16 >> 2);
      const int r = 16 * ((lane >> 4) & 1) + 4 * (l16 & 3), c = r0 + (decltype(is_q)::value ? ffn_q_order(r) : r);
      const unsigned char* a = tile + k * (BR * 2) + (((c >> 3) ^ L::key_across(k)) << 4) + (c & 7) * 2;
      struct { s16x4 lo, hi; } both = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a),
                                       __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + 4 * BR * 2))};
      return __builtin_bit_cast(v4i, both);
    } else {
      const int k = ks * L::KSTEP + 4 * h, c = r0 + (decltype(is_q)::value ? ffn_q_order(l32) : l32);
      v4i f;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        f[e] = *reinterpret_cast<const int*>(tile + (k + e) * (BR * 4) + (((c >> 2) ^ L::key_across(k)) << 4) + (c & 3) * 4);
      return f;
    }
  };

  floatx16 acc[MI][NI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[mi][ni][v] = 0.0f;

  struct Step { v4i p[MI], q[NI]; };                           // operands of KSTEP entries of k
  auto read_step = [&](int stage, int ks, Step& f) {
    const unsigned char* tp = smem + stage * STAGE;
    const unsigned char* tq = tp + P_BYTES;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
      f.p[mi] = fragment(std::bool_constant<P_ALONG>{}, std::false_type{}, tp, std::integral_constant<int, BM>{}, (wm * MI + mi) * 32, ks);
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
      const int r0 = GATED ? (ni < HALF ? (wn * HALF + ni) * 32 : COLS + (wn * HALF + ni - HALF) * 32) : (wn * NI + ni) * 32;
      f.q[ni] = fragment(std::bool_constant<Q_ALONG>{}, std::true_type{}, tq, std::integral_constant<int, BN>{}, r0, ks);
    }
  };
  // the products of a step; job(i) behind the i-th
  auto multiply = [&](const Step& f, auto&& job) {
    ffn_for<0, MI * NI>([&](auto i) {
      constexpr int I = decltype(i)::value;
      E::mma(acc[I / NI][I % NI], f.q[I % NI], f.p[I / NI]);
      job(i);
    });
  };
  auto no_job = [](auto) {};

  constexpr int STRETCH = kFfnList / BK;                       // K tiles of a stretch of the list
  auto renew_list = [&](int kt) {                              // called by all, before anything of K tile kt is asked for
    if constexpr (LISTED) {
      if (list && (kt - kt_lo) % STRETCH == 0) {
        __syncthreads();
        stretch(kt);
        __syncthreads();
      }
    }
  };
  if constexpr (ALIGNED) {
    // Two tiles in LDS.  A tile has four steps, whose operands are read one step ahead, the first step's under the products of the last
    // one of the tile before: by then all wavefronts have met, the tile has landed, and the one before is in registers, so that its
    // place takes the tile after next.  Its transfers are asked for one at a time between products, since a wavefront that asks for
    // several waits while the address unit takes them.
    constexpr int JOBS = JP + JQ, EACH = (JOBS + MI * NI - 1) / (MI * NI);      // transfers behind a product
    auto ask = [&](int kt, int stage) {
      renew_list(kt);
      look_up(kt);
      const Ask a = prepare(kt, stage);
      ffn_for<0, JOBS>([&](auto j) { request_one(a, j); });
    };
    if (kt_lo < kt_hi) ask(kt_lo, 0);
    if (kt_lo + 1 < kt_hi) {
      ask(kt_lo + 1, 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(JOBS) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    Step f0, f1;
    if (kt_lo < kt_hi) read_step(0, 0, f0);
    for (int kt = kt_lo; kt < kt_hi; ++kt) {
      const int stage = (kt - kt_lo) & 1;
      read_step(stage, 1, f1);
      __builtin_amdgcn_sched_barrier(0);
      multiply(f0, no_job);
      __builtin_amdgcn_sched_barrier(0);
      read_step(stage, 2, f0);
      __builtin_amdgcn_sched_barrier(0);
      multiply(f1, no_job);
      __builtin_amdgcn_sched_barrier(0);
      read_step(stage, 3, f1);
      __builtin_amdgcn_sched_barrier(0);
      multiply(f0, no_job);
      __builtin_amdgcn_sched_barrier(0);
      // the next tile has landed, and this one has been read, for every wavefront
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      // (behind the last tile but one, the last again, which nobody reads: a branch here would cost registers)
      const int ahead = min(kt + 2, kt_hi - 1);
      if (kt + 2 < kt_hi) renew_list(ahead);
      look_up(ahead);
      const Ask a = prepare(ahead, stage);
      read_step(stage ^ 1, 0, f0);
      __builtin_amdgcn_sched_barrier(0);
      multiply(f1, [&](auto i) {
        constexpr int I = decltype(i)::value;
        __builtin_amdgcn_sched_barrier(0);
        ffn_for<I * EACH, (I + 1) * EACH < JOBS ? (I + 1) * EACH : JOBS>([&](auto j) { request_one(a, j); });
        __builtin_amdgcn_sched_barrier(0);
      });
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // nothing may still be on its way into LDS when the workgroup ends
  } else {
    if (kt_lo < kt_hi) {
      renew_list(kt_lo);
      hold(kt_lo);
    }
    for (int kt = kt_lo; kt < kt_hi; ++kt) {
      __syncthreads();
      put();
      __syncthreads();
      if (kt + 1 < kt_hi) {
        renew_list(kt + 1);
        hold(kt + 1);
      }
#pragma unroll
      for (int ks = 0; ks < L::STEPS; ++ks) {
        Step f;
        read_step(0, ks, f);
        multiply(f, no_job);
      }
    }
  }

  // ---- results: the lane has row l32 of a block, its columns 16 h .. 16 h + 15 ----
  const int n = p.n, m = p.m;
  auto store = [&](T* c, int64_t ldc, int row, int col, const floatx16& v) {      // row < 0: none
    if constexpr (ALIGNED) {
      store_block_pairs<DT, false>(v, row, false, col, c, nullptr, 0, (int)ldc);
    } else if (row >= 0) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (col + e < n) c[(int64_t)row * ldc + col + e] = E::from_float(v[e]);
    }
  };
  auto load16 = [&](const T* c, int64_t ldc, int row, int col, float (&out)[16]) {
    const T* s = c + (int64_t)row * ldc + col;
#pragma unroll
    for (int g = 0; g < 16 / V; ++g) {
      const v4i q = load_group(s + g * V, row < 0 ? 0 : n - col - g * V);
      T e[V];
      __builtin_memcpy(e, &q, 16);
#pragma unroll
      for (int i = 0; i < V; ++i) out[g * V + i] = (float)e[i];
    }
  };
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) {
    const int i = m0 + (wm * MI + mi) * 32 + l32;
    const int row = i < m ? i : -1;
    int out_row = row;
    if (row >= 0 && p.c_rows) out_row = p.c_rows[row];
#pragma unroll
    for (int ni = 0; ni < HALF; ++ni) {
      const int col = n0 + (wn * HALF + ni) * 32 + 16 * h;
      if constexpr (WHAT == kFfnUp) {
        floatx16 hidden;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float a, da;
          ffn_act(p.activation, acc[mi][ni][e], a, da);
          hidden[e] = a * acc[mi][ni + HALF][e];
        }
        store(static_cast<T*>(p.c[0]), p.ldc, row, col, hidden);
        if (p.saved) {
          T* g = static_cast<T*>(p.saved);
          store(g, p.ldc, row, col, acc[mi][ni]);
          store(g + (int64_t)m * n, p.ldc, row, col, acc[mi][ni + HALF]);
        }
      } else if constexpr (WHAT == kFfnGateGrad) {
        float g[16], u[16];
        const T* sv = static_cast<const T*>(p.saved);
        load16(sv, p.ldc, row, col, g);
        load16(sv + (int64_t)m * n, p.ldc, row, col, u);
        floatx16 dg, du;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float a, da;
          ffn_act(p.activation, g[e], a, da);
          dg[e] = acc[mi][ni][e] * u[e] * da;
          du[e] = acc[mi][ni][e] * a;
        }
        store(static_cast<T*>(p.c[0]), p.ldc, row, col, dg);
        store(static_cast<T*>(p.c[1]), p.ldc, row, col, du);
      } else {
        if (WHAT == kFfnWGrad && p.splits > 1) {
          if (row >= 0) {
            float* dst = p.partial + (((int64_t)z * p.splits + split) * m + row) * n + col;
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (col + e < n) dst[e] = acc[mi][ni][e];
          }
        } else {
          store(static_cast<T*>(p.c[z]), p.ldc, out_row, col, acc[mi][ni]);
        }
      }
    }
  }
}

template <int DT, bool P_ALONG, bool Q_ALONG, int WHAT, int BM, int BN, int WAVES_M, int WAVES_N, bool ALIGNED>
hipError_t ffn_launch_tile(FfnGemm g, hipStream_t s) {
  auto kernel = ffn_gemm_kernel<DT, P_ALONG, Q_ALONG, WHAT, BM, BN, WAVES_M, WAVES_N, ALIGNED>;
  constexpr int cols = WHAT == kFfnUp ? BN / 2 : BN;
  g.m_tiles = (g.m + BM - 1) / BM;
  g.n_tiles = (g.n + cols - 1) / cols;
  g.group = 8;
  const bool listed = WHAT == kFfnWGrad && (g.p_rows || g.q_rows);
  const int lds = (BM + BN) * 128 * (ALIGNED ? 2 : 1) + (listed ? kFfnList * 4 : 0);
  static std::atomic<uint64_t> told{0};
  const hipError_t e = ffn_allow_lds(reinterpret_cast<const void*>(kernel), (BM + BN) * 128 * (ALIGNED ? 2 : 1) + kFfnList * 4, told);
  if (e != hipSuccess) return e;
  const int64_t total = (int64_t)g.m_tiles * g.n_tiles * g.batch * g.splits;
  kernel<<<dim3((unsigned)((total + 7) / 8 * 8)), dim3(64 * WAVES_M * WAVES_N), lds, s>>>(g);
  return hipGetLastError();
}

template <int DT, bool P_ALONG, bool Q_ALONG, int WHAT>
hipError_t ffn_launch_what(const FfnGemm& g, int tile, bool aligned, hipStream_t s) {
  if (!aligned) return ffn_launch_tile<DT, P_ALONG, Q_ALONG, WHAT, 128, 128, 2, 2, false>(g, s);
  if (tile == 1) return ffn_launch_tile<DT, P_ALONG, Q_ALONG, WHAT, 256, 256, 2, 4, true>(g, s);
  return ffn_launch_tile<DT, P_ALONG, Q_ALONG, WHAT, 128, 128, 2, 2, true>(g, s);
}

template <int DT> hipError_t ffn_launch_type(FfnProduct what, const FfnGemm& g, int tile, bool aligned, hipStream_t s) {
  switch (what) {
    case kFfnUp: return ffn_launch_what<DT, true, true, kFfnUp>(g, tile, aligned, s);
    case kFfnDown: return ffn_launch_what<DT, true, true, kFfnDown>(g, tile, aligned, s);
    case kFfnGateGrad: return ffn_launch_what<DT, true, false, kFfnGateGrad>(g, tile, aligned, s);
    case kFfnInGrad: return ffn_launch_what<DT, true, false, kFfnInGrad>(g, tile, aligned, s);
    case kFfnWGrad: return ffn_launch_what<DT, false, false, kFfnWGrad>(g, tile, aligned, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace sc
