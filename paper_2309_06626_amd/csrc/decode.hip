// Attention of single tokens over a paged cache: calls (the kernels are in decode_kernel.hpp).
#include "../../include/sparse_attention.h"

#include "conv_params.hpp"
#include "decode_params.hpp"

#include <algorithm>

namespace sc {

void note_hip_error(int32_t code);
int32_t kv_entries(const sc_kv_desc* d);
sc_status check_kv(const sc_kv_desc* d);
sc_status check_attn(const sc_attn_desc* d);

static int decode_width(int d) { return d <= 64 ? 64 : 128; }

// Stretches of the longest sequence that the table allows; how long the sequences are is known on the device alone.  A workgroup of entries above 64
// channels fills a compute unit's LDS, of codes of 16-bit types two do.  (Two of 16-bit entries of up to 64 channels would fit as well; they are counted as
// those above.)  Few sequences: as many stretches as run at once (100 000 rows, 8 key-value heads: 32 stretches 79 us, 64 89, 96 100; 33 sequences of up
// to 4 000 rows in 8 bits, 4 heads: 2 39 us, 4 29.7, 6 32).  Many, whose lengths differ: three times as many (64 sequences of 4 096 to 8 192 rows, 8
// heads: 1 316 us, 2 306, 4 304).  Between the two, where the number of stretches jumps from 2 to 6, nothing was measured.  A stretch has a tile for each
// wavefront at least, and no more pages than a workgroup holds.
static int64_t decode_splits(const sc_attn_desc* d, const sc_kv_desc* cache, int64_t rows, int64_t table_width) {
  const int64_t blocks = (d->heads / d->kv_heads + 31) / 32, base = std::max<int64_t>(rows * blocks * d->kv_heads, 1);
  int64_t keys = table_width * cache->page_rows;
  // (a window that covers whole pages, and the tile that it ends in)
  if (d->window && d->window < keys - 64) keys = d->window + 64;
  const int64_t tiles = (keys + 31) / 32;
  const int64_t together = cache->bits == 8 && cache->dtype != SC_F32 ? 512 : 256;
  int64_t splits = 2 * base <= together ? (4 * together / base + 1) / 4 : (3 * together + base - 1) / base;
  splits = std::min(splits, (tiles + kDecodeWaves - 1) / kDecodeWaves);
  splits = std::max<int64_t>(splits, 1);
  // pages of a stretch: those of its tiles, rounded up, and one it begins within
  while ((((tiles + splits - 1) / splits + kDecodeWaves) * 32) / cache->page_rows + 2 > kDecodePages) splits += (splits + 3) / 4;
  return splits;
}

static sc_status decode_check(const sc_attn_desc* desc, const sc_kv_desc* cache, int64_t rows, int64_t table_width) {
  sc_status st = check_attn(desc);
  if (st == SC_OK) st = check_kv(cache);
  if (st != SC_OK) return st;
  if (desc->dtype != cache->dtype || desc->kv_heads != cache->kv_heads || desc->d != cache->d) return SC_ERR_BAD_SHAPE;
  if (rows < 0 || table_width < 0 || rows > (1 << 24) || table_width > 0x7fffffff || table_width * cache->page_rows > 0x7fffffff) return SC_ERR_BAD_SHAPE;
  // a launch has fewer than 2^32 lanes
  const int64_t blocks = (desc->heads / desc->kv_heads + 31) / 32;
  if (rows * blocks * desc->kv_heads * decode_splits(desc, cache, rows, table_width) >= (1 << 24) || rows * desc->heads >= (1 << 24)) return SC_ERR_BAD_SHAPE;
  return SC_OK;
}

static size_t decode_up(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace sc

extern "C" {

sc_status sparse_attn_decode_workspace_bytes(const sc_attn_desc* desc, const sc_kv_desc* cache, int64_t rows, int64_t table_width,
                                             size_t* bytes) {
  if (!bytes) return SC_ERR_NULL;
  *bytes = 0;
  const sc_status st = sc::decode_check(desc, cache, rows, table_width);
  if (st != SC_OK) return st;
  const int64_t splits = sc::decode_splits(desc, cache, rows, table_width), shares = splits > 1 ? rows * desc->heads * splits : 0;
  *bytes = 256 + sc::decode_up((size_t)shares * sc::decode_width(desc->d) * 4) + sc::decode_up((size_t)shares * 8);
  return SC_OK;
}

sc_status sparse_attn_decode(const sc_attn_desc* desc, const sc_kv_desc* cache, int64_t rows, const void* q_dev, const int32_t* table_dev,
                             int64_t table_width, const int32_t* lengths_dev, const void* k_pages_dev, const void* v_pages_dev,
                             const float* k_scales_dev, const float* v_scales_dev, void* o_dev, void* workspace_dev,
                             size_t workspace_bytes, void* hip_stream) {
  const sc_status st = sc::decode_check(desc, cache, rows, table_width);
  if (st != SC_OK) return st;
  if (rows > 0 && (!q_dev || !o_dev || !lengths_dev || (table_width > 0 && !table_dev))) return SC_ERR_NULL;
  if (!k_pages_dev || !v_pages_dev || !workspace_dev || (cache->bits == 8 && (!k_scales_dev || !v_scales_dev))) return SC_ERR_NULL;
  size_t need = 0;
  sparse_attn_decode_workspace_bytes(desc, cache, rows, table_width, &need);
  if (workspace_bytes < need) return SC_ERR_WORKSPACE;
  if (((uintptr_t)q_dev | (uintptr_t)table_dev | (uintptr_t)lengths_dev | (uintptr_t)k_pages_dev | (uintptr_t)v_pages_dev | (uintptr_t)k_scales_dev |
       (uintptr_t)v_scales_dev | (uintptr_t)o_dev | (uintptr_t)workspace_dev) & 15)
    return SC_ERR_ALIGN;
  if (rows == 0) return SC_OK;
  const int eb = desc->dtype == SC_F32 ? 4 : 2;
  sc::DecodeParams p = {};
  p.q = q_dev;
  p.k_pages = k_pages_dev;
  p.v_pages = v_pages_dev;
  p.k_scales = k_scales_dev;
  p.v_scales = v_scales_dev;
  p.o = o_dev;
  p.table = table_dev;
  p.lengths = lengths_dev;
  p.rows = rows;
  p.table_width = table_width;
  p.heads = desc->heads;
  p.kv_heads = desc->kv_heads;
  p.d = desc->d;
  p.pages = cache->pages;
  p.shift = __builtin_ctz(cache->page_rows);
  p.row_bytes = sc::kv_entries(cache) * (cache->bits == 8 ? 1 : eb);
  p.window = desc->window;
  p.splits = (int32_t)sc::decode_splits(desc, cache, rows, table_width);
  p.blocks = (desc->heads / desc->kv_heads + 31) / 32;
  p.vec = desc->d * eb % 16 == 0;
  p.scale = desc->scale;
  p.part_o = static_cast<float*>(workspace_dev);
  p.part_m = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) +
                                      sc::decode_up((size_t)rows * p.heads * p.splits * sc::decode_width(p.d) * 4));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = desc->dtype == SC_BF16  ? sc::decode_launch<sc::kBF16>(p, cache->bits == 8, s)
                       : desc->dtype == SC_F16 ? sc::decode_launch<sc::kF16>(p, cache->bits == 8, s)
                                               : sc::decode_launch<sc::kF32>(p, cache->bits == 8, s);
  if (e != hipSuccess) { sc::note_hip_error((int32_t)e); return SC_ERR_HIP; }
  return SC_OK;
}

}  // extern "C"
