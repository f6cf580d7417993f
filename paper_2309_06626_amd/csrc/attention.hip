// Attention over packed sequences of kept rows: plans and calls (the kernels are in attn_kernel.hpp).
//
// A plan is a list of a workgroup's shares: tiles of packed rows (forward, and the queries' gradient) and of keys (their and the values'
// gradient) of every sequence, those with the most to do first.
#include "../../include/sparse_attention.h"

#include "attn_params.hpp"
#include "conv_params.hpp"
#include "rows.hpp"

#include <algorithm>
#include <cmath>
#include <vector>

struct sc_attn {
  sc_attn_desc desc;
  int64_t end, kept;               // rows of the sequences, and how many of them are kept
  uint64_t version;                // of the row set; 0: none
  sc::AttnTiles forward, backward;
  const sc::AttnItem* items[3];    // of the forward pass, the queries' gradient, and that of keys and values
  int32_t n_items[3];
};

namespace sc {

void note_hip_error(int32_t code);

static hipError_t attn_dispatch(int dtype, int what, const AttnParams& p, AttnTiles t, int vec, hipStream_t s) {
  if (t.waves == 1) {
    if (dtype == SC_BF16) return attn_few_launch<kBF16>(what, p, vec, s);
    if (dtype == SC_F16) return attn_few_launch<kF16>(what, p, vec, s);
    return attn_few_launch<kF32>(what, p, vec, s);
  }
  if (dtype == SC_BF16) return attn_launch<kBF16>(what, p, t, vec, s);
  if (dtype == SC_F16) return attn_launch<kF16>(what, p, t, vec, s);
  return attn_launch<kF32>(what, p, t, vec, s);
}

// kept rows before each start
__global__ __launch_bounds__(256) void attn_starts_kernel(const int32_t* __restrict__ starts, int n, const int32_t* __restrict__ row_idx,
                                                          int32_t kept, int32_t* __restrict__ out) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  int lo = 0, hi = kept;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (row_idx[mid] < starts[i]) lo = mid + 1;
    else hi = mid;
  }
  out[i] = lo;
}

// Zeros in the dropped rows of up to three outputs (of null and 0 bytes where there are fewer).
static void attn_zeros_of(const sc_rows* set, int64_t rows, std::initializer_list<void*> out, std::initializer_list<int64_t> stride,
                          std::initializer_list<int64_t> width, AttnZeros* z) {
  *z = {};
  if (!set || set->kept == set->rows || rows == 0) return;
  z->slot = set->kept ? set->slot : nullptr;
  z->rows = rows;
  std::copy(out.begin(), out.end(), z->out);
  std::copy(stride.begin(), stride.end(), z->stride);
  std::copy(width.begin(), width.end(), z->width);
  uint64_t all = 0;
  for (int k = 0; k < 3; ++k) all |= (uint64_t)(uintptr_t)z->out[k] | (uint64_t)z->stride[k] | (uint64_t)z->width[k];
  z->vec = all % 16 == 0;
  z->blocks = (int32_t)std::min<int64_t>((rows + 31) / 32, 512);
}

static size_t attn_up(size_t n) { return (n + 255) & ~(size_t)255; }
static int64_t attn_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int kAttnRowsLeast = 128;      // packed rows of the smallest tile
constexpr int kAttnFew = 2048;           // most workgroups of the tiles for few rows

sc_status check_attn(const sc_attn_desc* d) {
  if (!d) return SC_ERR_NULL;
  if (d->dtype != SC_F32 && d->dtype != SC_F16 && d->dtype != SC_BF16) return SC_ERR_UNSUPPORTED;
  if (d->causal != 0 && d->causal != 1) return SC_ERR_UNSUPPORTED;
  if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads != 0 || d->heads / d->kv_heads > 512 || d->heads > (1 << 20)) return SC_ERR_BAD_SHAPE;
  if (d->d < 1 || d->window < 0 || !std::isfinite(d->scale) || !(d->scale > 0.0f) || d->scale > 0x1p127f) return SC_ERR_BAD_SHAPE;      // (kernels take it in exponents of 2)
  if (d->d > 128) return SC_ERR_UNSUPPORTED;
  return SC_OK;
}

// (bytes of the starts twice, of the items of rows and of keys)
struct AttnLayout { size_t starts, row_items, key_items; };
static AttnLayout attn_layout(const sc_attn_desc* d, int64_t seqs, int64_t rows) {
  const int64_t group = d->heads / d->kv_heads;
  AttnLayout l;
  l.starts = attn_up((size_t)(seqs + 1) * 4);
  l.row_items = attn_up((size_t)(rows * group / kAttnRowsLeast + seqs + kAttnFew) * sizeof(AttnItem));      // (twice: forward and backward)
  l.key_items = attn_up((size_t)(rows / (32 * kAttnKeyWaves) + seqs + kAttnFew) * sizeof(AttnItem));
  return l;
}

// Tiles of `per` packed rows of every sequence, longest first.
// Returns what a tile sees on average.
static int64_t attn_items(const std::vector<int32_t>& starts, const sc_attn_desc& d, int64_t per, bool keys, std::vector<AttnItem>& items) {
  const int64_t group = keys ? 1 : d.heads / d.kv_heads;
  items.clear();
  std::vector<int64_t> work;
  for (size_t s = 0; s + 1 < starts.size(); ++s) {
    const int64_t n = starts[s + 1] - starts[s], tiles = attn_ceil(n * group, per);
    for (int64_t t = 0; t < tiles; ++t) {
      const int64_t lo = t * per / group, hi = std::min((t * per + per - 1) / group, n - 1);      // rows (or keys) of the tile
      int64_t first = 0, last = n - 1;                                                           // and what they see (or are seen by)
      if (d.window) {
        first = std::max<int64_t>(0, lo - d.window + 1);
        last = std::min<int64_t>(last, hi + d.window - 1);
      }
      if (d.causal) (keys ? first : last) = keys ? lo : hi;
      work.push_back(last - first + 1);
      items.push_back({starts[s], (int32_t)n, (int32_t)t, 0});
    }
  }
  std::vector<int32_t> order(items.size());
  for (size_t i = 0; i < order.size(); ++i) order[i] = (int32_t)i;
  std::stable_sort(order.begin(), order.end(), [&](int32_t a, int32_t b) { return work[a] > work[b]; });
  std::vector<AttnItem> sorted(items.size());
  for (size_t i = 0; i < order.size(); ++i) sorted[i] = items[order[i]];
  items.swap(sorted);
  int64_t all = 0;
  for (int64_t w : work) all += w;
  return work.empty() ? 0 : all / (int64_t)work.size();
}

static sc_status attn_plan(sc_attn* plan, int64_t seqs, const int64_t* starts, const sc_rows* set, unsigned char* w, hipStream_t s) {
  const AttnLayout l = attn_layout(&plan->desc, seqs, plan->end);
  std::vector<int32_t> at(seqs + 1);
  for (int64_t i = 0; i <= seqs; ++i) at[i] = (int32_t)starts[i];
  hipError_t e = hipSuccess;
  if (set && set->kept != set->rows && plan->end > 0) {
    std::vector<int32_t> kept(at.size());      // (before the copies: what throws between them and the wait would give back memory that they use)
    int32_t *in = reinterpret_cast<int32_t*>(w), *out = reinterpret_cast<int32_t*>(w + l.starts);
    e = hipMemcpyAsync(in, at.data(), at.size() * 4, hipMemcpyHostToDevice, s);
    if (e == hipSuccess) {
      attn_starts_kernel<<<dim3((unsigned)(at.size() + 255) / 256), dim3(256), 0, s>>>(in, (int)at.size(), set->row_idx, (int32_t)set->kept, out);
      e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipMemcpyAsync(kept.data(), out, kept.size() * 4, hipMemcpyDeviceToHost, s);
    const hipError_t waited = hipStreamSynchronize(s);      // (also after an error: the copies read and write these vectors)
    if (e == hipSuccess) e = waited;
    at.swap(kept);
  }
  if (e != hipSuccess) { note_hip_error((int32_t)e); return SC_ERR_HIP; }
  plan->kept = at.back();
  // Workgroups of eight wavefronts read keys and values half as often; those of four leave less undone at a sequence's ends, and two run on a
  // compute unit side by side (8 192 rows that see 4 096 on average: 494 and 510 us; 23 sequences, window 1 024: 145 and 136).  The queries' gradient
  // has LDS for one of either: eight where they are filled (4 x 2 048 rows: 346 and 370 us).  Narrow heads of short sequences take tiles of
  // 32 keys, whose registers allow three workgroups (64 x 98 rows, 12 heads of 64: 15.1 and 18 us; 16 x 1 024: 77 and 75).
  const sc_attn_desc& d = plan->desc;
  const bool wide = d.dtype != SC_F32;
  std::vector<AttnItem> items[3];
  const int64_t seen = attn_items(at, d, 128, false, items[0]);
  plan->forward = {wide && seen >= 2048 ? 8 : 4, d.d <= 64 && seen <= 256 ? 32 : 64};
  plan->backward = {wide && d.d % 8 == 0 && plan->kept * (d.heads / d.kv_heads) >= 512 * seqs ? 8 : 4, 64};
  // Few rows: tiles of 32, whose workgroup's wavefronts share what passes by.  Gradients up to 1 024 workgroups (16 heads on 4: 2 048 rows of 128 in
  // 16 bits, training 367 and 235 us, 16 x 128 rows 50.9 and 49.3; 8 heads of 64 floats: 512 rows 175 and 93, 8 x 512 184 and 159, 16 x 512 253 and
  // 269), of long sequences in 16 bits up to 2 048 (4 096 rows 734 and 591, 32 x 128 rows 63 and 83).  Forward of floats alone, up to 512, where it takes
  // those 93 us to 71 (8 x 512, 1 024 workgroups of heads of 128: 343 and 364); in 16 bits it gains nothing (1 024 rows alone: 21 and 33).
  int64_t row_tiles = 0, key_tiles = 0;
  for (int64_t i = 0; i < seqs; ++i) {
    row_tiles += attn_ceil((int64_t)(at[i + 1] - at[i]) * (d.heads / d.kv_heads), 32);
    key_tiles += attn_ceil(at[i + 1] - at[i], 32);
  }
  const bool few = row_tiles * d.kv_heads <= 512 && !wide, few_backward = std::max(row_tiles, key_tiles) * d.kv_heads <= (wide && seen >= 1024 ? kAttnFew : 1024);
  if (few) plan->forward.waves = 1;
  if (few_backward) plan->backward.waves = 1;
  if (plan->forward.waves != 4) attn_items(at, d, 32 * plan->forward.waves, false, items[0]);
  attn_items(at, d, 32 * plan->backward.waves, false, items[1]);
  attn_items(at, d, few_backward ? 32 : 32 * kAttnKeyWaves, true, items[2]);
  unsigned char* to = w + 2 * l.starts;
  for (int k = 0; k < 3; ++k) {
    plan->items[k] = reinterpret_cast<const AttnItem*>(to);
    plan->n_items[k] = (int32_t)items[k].size();
    if (e == hipSuccess && !items[k].empty()) e = hipMemcpyAsync(to, items[k].data(), items[k].size() * sizeof(AttnItem), hipMemcpyHostToDevice, s);
    to += k < 2 ? l.row_items : l.key_items;
  }
  if (!items[0].empty()) {
    const hipError_t waited = hipStreamSynchronize(s);
    if (e == hipSuccess) e = waited;
  }
  if (e != hipSuccess) { note_hip_error((int32_t)e); return SC_ERR_HIP; }
  return SC_OK;
}

// what runs and backward passes check alike
static sc_status attn_check_call(const sc_attn* plan, const sc_rows* rows, int32_t row_format) {
  if (!plan) return SC_ERR_NULL;
  if (row_format != SC_ROWS_DENSE && row_format != SC_ROWS_COMPACT) return SC_ERR_UNSUPPORTED;
  if ((rows != nullptr) != (plan->version != 0)) return SC_ERR_BAD_SHAPE;
  if (rows && rows->version != plan->version) return SC_ERR_MASK_COUNT;
  return SC_OK;
}

struct AttnMatrix { const void* at; int64_t stride; int32_t heads; };      // [rows][heads][d]

static sc_status attn_check_matrices(const sc_attn* plan, std::initializer_list<AttnMatrix> ms, int* vec) {
  const int eb = plan->desc.dtype == SC_F32 ? 4 : 2;
  uint64_t all = (uint64_t)plan->desc.d * eb;
  for (const AttnMatrix& m : ms) {
    if (plan->kept > 0 && !m.at) return SC_ERR_NULL;
    if (m.stride < (int64_t)m.heads * plan->desc.d || m.stride > ((int64_t)1 << 40)) return SC_ERR_BAD_SHAPE;
    if ((uintptr_t)m.at % eb) return SC_ERR_ALIGN;
    all |= (uint64_t)(uintptr_t)m.at | (uint64_t)m.stride * eb;
  }
  *vec = all % 16 == 0 ? 2 : all % 4 == 0 ? 1 : 0;
  return SC_OK;
}

static AttnParams attn_params(const sc_attn* plan, const sc_rows* rows, int32_t row_format) {
  const sc_attn_desc& d = plan->desc;
  AttnParams p = {};
  p.map = row_format == SC_ROWS_DENSE && rows && rows->kept != rows->rows ? rows->row_idx : nullptr;
  p.heads = d.heads;
  p.kv_heads = d.kv_heads;
  p.group = d.heads / d.kv_heads;
  p.d = d.d;
  p.causal = d.causal;
  p.window = d.window;
  p.magic = ((1u << 20) + p.group - 1) / p.group;
  p.scale = d.scale;
  return p;
}

}  // namespace sc

extern "C" {

sc_status sparse_attn_workspace_bytes(const sc_attn_desc* desc, int64_t seqs, int64_t rows, size_t* bytes) {
  if (!bytes) return SC_ERR_NULL;
  *bytes = 0;
  const sc_status st = sc::check_attn(desc);
  if (st != SC_OK) return st;
  // packed rows are counted in 32 bits, of which tiles need a few; a launch of workgroups of 512 lanes, those of zeros among them, has fewer than 2^32
  if (seqs < 0 || rows < 0 || seqs > (1 << 24) || rows > 0x7fffffff || rows * desc->heads > ((int64_t)1 << 36) ||
      rows * (desc->heads / desc->kv_heads) > (1 << 30) || (rows * (desc->heads / desc->kv_heads) / sc::kAttnRowsLeast + seqs) * desc->kv_heads >= (1 << 23) - 512)
    return SC_ERR_BAD_SHAPE;
  const sc::AttnLayout l = sc::attn_layout(desc, seqs, rows);
  *bytes = 2 * l.starts + 2 * l.row_items + l.key_items;
  return SC_OK;
}

sc_status sparse_attn_plan(const sc_attn_desc* desc, int64_t seqs, const int64_t* starts, const sc_rows* rows, void* workspace_dev,
                           size_t workspace_bytes, void* hip_stream, sc_attn** out) {
  if (!out) return SC_ERR_NULL;
  *out = nullptr;
  sc_status st = sc::check_attn(desc);
  if (st != SC_OK) return st;
  if (!starts || !workspace_dev) return SC_ERR_NULL;
  if (seqs < 0 || seqs > (1 << 24) || starts[0] != 0) return SC_ERR_BAD_SHAPE;
  for (int64_t i = 0; i < seqs; ++i)
    if (starts[i + 1] < starts[i]) return SC_ERR_BAD_SHAPE;
  if (rows && starts[seqs] > rows->rows) return SC_ERR_BAD_SHAPE;
  size_t need = 0;
  st = sparse_attn_workspace_bytes(desc, seqs, starts[seqs], &need);
  if (st != SC_OK) return st;
  if (workspace_bytes < need) return SC_ERR_WORKSPACE;
  if ((uintptr_t)workspace_dev & 15) return SC_ERR_ALIGN;
  sc_attn* plan = nullptr;
  try {      // the lists on the host
    plan = new sc_attn;
    plan->desc = *desc;
    plan->end = starts[seqs];
    plan->version = rows ? rows->version : 0;
    st = sc::attn_plan(plan, seqs, starts, rows, static_cast<unsigned char*>(workspace_dev), static_cast<hipStream_t>(hip_stream));
  } catch (...) {      // (there is no memory for them)
    sc::note_hip_error((int32_t)hipErrorOutOfMemory);
    st = SC_ERR_HIP;
  }
  if (st != SC_OK) {
    delete plan;
    return st;
  }
  *out = plan;
  return SC_OK;
}

sc_status sparse_attn_info(const sc_attn* plan, int64_t* end, int64_t* kept) {
  if (!plan) return SC_ERR_NULL;
  if (end) *end = plan->end;
  if (kept) *kept = plan->kept;
  return SC_OK;
}

void sparse_attn_destroy(sc_attn* plan) { delete plan; }

sc_status sparse_attn_run(const sc_attn* plan, const sc_rows* rows, int32_t row_format, const void* q_dev, int64_t q_stride,
                          const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride, void* o_dev, float* lse_dev,
                          void* hip_stream) {
  sc_status st = sc::attn_check_call(plan, rows, row_format);
  if (st != SC_OK) return st;
  const sc_attn_desc& d = plan->desc;
  int vec;
  st = sc::attn_check_matrices(plan, {{q_dev, q_stride, d.heads}, {k_dev, k_stride, d.kv_heads}, {v_dev, v_stride, d.kv_heads}}, &vec);
  if (st != SC_OK) return st;
  if (plan->end > 0 && !o_dev && (plan->kept > 0 || row_format == SC_ROWS_DENSE)) return SC_ERR_NULL;
  if (((uintptr_t)o_dev | (uintptr_t)lse_dev) & 15) return SC_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  sc::AttnParams p = sc::attn_params(plan, rows, row_format);
  p.q = q_dev;
  p.k = k_dev;
  p.v = v_dev;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.out = o_dev;
  p.lse = lse_dev;
  p.items = plan->items[0];
  p.n_items = plan->n_items[0];
  hipError_t e = hipSuccess;
  if (row_format == SC_ROWS_DENSE) {
    const int64_t width = (int64_t)d.heads * d.d * (d.dtype == SC_F32 ? 4 : 2);
    sc::attn_zeros_of(rows, plan->end, {o_dev}, {width}, {width}, &p.zeros);
  }
  if (p.n_items > 0 || p.zeros.blocks > 0) e = sc::attn_dispatch(d.dtype, sc::kAttnForward, p, plan->forward, vec, s);
  if (e != hipSuccess) { sc::note_hip_error((int32_t)e); return SC_ERR_HIP; }
  return SC_OK;
}

sc_status sparse_attn_backward_workspace_bytes(const sc_attn* plan, size_t* bytes) {
  if (!bytes) return SC_ERR_NULL;
  *bytes = 0;
  if (!plan) return SC_ERR_NULL;
  *bytes = 256 + 2 * sc::attn_up((size_t)plan->kept * plan->desc.heads * 4);
  return SC_OK;
}

sc_status sparse_attn_backward(const sc_attn* plan, const sc_rows* rows, int32_t row_format, const void* q_dev, int64_t q_stride,
                               const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride, const void* o_dev,
                               const float* lse_dev, const void* do_dev, void* dq_dev, int64_t dq_stride, void* dk_dev,
                               int64_t dk_stride, void* dv_dev, int64_t dv_stride, void* workspace_dev, size_t workspace_bytes,
                               void* hip_stream) {
  sc_status st = sc::attn_check_call(plan, rows, row_format);
  if (st != SC_OK) return st;
  const sc_attn_desc& d = plan->desc;
  int vec;
  st = sc::attn_check_matrices(plan, {{q_dev, q_stride, d.heads}, {k_dev, k_stride, d.kv_heads}, {v_dev, v_stride, d.kv_heads},
                                      {dq_dev, dq_stride, d.heads}, {dk_dev, dk_stride, d.kv_heads}, {dv_dev, dv_stride, d.kv_heads}}, &vec);
  if (st != SC_OK) return st;
  if (plan->end > 0 && row_format == SC_ROWS_DENSE && (!dq_dev || !dk_dev || !dv_dev)) return SC_ERR_NULL;
  if (plan->kept > 0 && (!o_dev || !lse_dev || !do_dev)) return SC_ERR_NULL;
  if (!workspace_dev) return SC_ERR_NULL;
  size_t need = 0;
  sparse_attn_backward_workspace_bytes(plan, &need);
  if (workspace_bytes < need) return SC_ERR_WORKSPACE;
  if (((uintptr_t)o_dev | (uintptr_t)lse_dev | (uintptr_t)do_dev | (uintptr_t)workspace_dev) & 15) return SC_ERR_ALIGN;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  sc::AttnParams p = sc::attn_params(plan, rows, row_format);
  p.q = q_dev;
  p.k = k_dev;
  p.v = v_dev;
  p.o = o_dev;
  p.d_o = do_dev;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.dq = dq_dev;
  p.dk = dk_dev;
  p.dv = dv_dev;
  p.dq_stride = dq_stride;
  p.dk_stride = dk_stride;
  p.dv_stride = dv_stride;
  p.lse = const_cast<float*>(lse_dev);
  p.stats[0] = static_cast<float*>(workspace_dev);
  p.stats[1] = p.stats[0] + sc::attn_up((size_t)plan->kept * d.heads * 4) / 4;
  p.items = plan->items[1];
  p.n_items = plan->n_items[1];
  if (row_format == SC_ROWS_DENSE) {
    const int64_t eb = d.dtype == SC_F32 ? 4 : 2, q = d.heads * eb * d.d, kv = d.kv_heads * eb * d.d;
    sc::attn_zeros_of(rows, plan->end, {dq_dev, dk_dev, dv_dev}, {dq_stride * eb, dk_stride * eb, dv_stride * eb}, {q, kv, kv}, &p.zeros);
  }
  hipError_t e = hipSuccess;
  if (p.n_items > 0 || p.zeros.blocks > 0) e = sc::attn_dispatch(d.dtype, sc::kAttnBackwardQ, p, plan->backward, vec, s);      // (leaves statistics for the keys)
  p.zeros.blocks = 0;
  p.items = plan->items[2];
  p.n_items = plan->n_items[2];
  if (e == hipSuccess && p.n_items > 0) e = sc::attn_dispatch(d.dtype, sc::kAttnBackwardKV, p, plan->backward, vec, s);
  if (e != hipSuccess) { sc::note_hip_error((int32_t)e); return SC_ERR_HIP; }
  return SC_OK;
}

}  // extern "C"
