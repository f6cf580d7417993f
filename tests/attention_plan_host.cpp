// The host's side of sparse_attn_plan with HIP calls of its own: copies are on their way until the stream is waited for, and the n-th
// allocation fails.  Prints, for n from 1 until none fails, whether memory was given back with a copy on its way from or to it, and what leaked.
#include "../include/sparse_attention.h"
#include "../paper_2309_06626_amd/csrc/attn_params.hpp"
#include "../paper_2309_06626_amd/csrc/conv_params.hpp"
#include "../paper_2309_06626_amd/csrc/rows.hpp"

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <new>
#include <vector>

static bool armed;
static long fail_at, asked, live, touched;
struct Range { const char *at; size_t bytes; };
static Range flying[64];
static int n_flying;
static std::map<void*, size_t>* sizes;

static void* take(size_t n) {
  if (armed && ++asked == fail_at) return nullptr;
  void* p = std::malloc(n ? n : 1);
  if (armed) {
    armed = false;
    (*sizes)[p] = n;
    armed = true;
    ++live;
  }
  return p;
}
static void give(void* p) {
  if (armed && p) {
    armed = false;
    const size_t n = (*sizes)[p];
    sizes->erase(p);
    for (int i = 0; i < n_flying; ++i)
      touched += flying[i].at < (char*)p + n && (char*)p < flying[i].at + flying[i].bytes;
    armed = true;
    --live;
  }
  std::free(p);
}
void* operator new(size_t n) {
  void* p = take(n);
  if (!p) throw std::bad_alloc();
  return p;
}
void* operator new(size_t n, const std::nothrow_t&) noexcept { return take(n); }
void operator delete(void* p) noexcept { give(p); }
void operator delete(void* p, size_t) noexcept { give(p); }
void operator delete(void* p, const std::nothrow_t&) noexcept { give(p); }

extern "C" {
hipError_t hipMemcpyAsync(void* to, const void* from, size_t n, hipMemcpyKind kind, hipStream_t) {
  std::memcpy(to, from, n);
  flying[n_flying++] = {static_cast<const char*>(kind == hipMemcpyHostToDevice ? from : to), n};
  return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) {
  n_flying = 0;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
// the only kernel of a plan: every second row is kept
hipError_t hipLaunchKernel(const void*, dim3, dim3, void** args, size_t, hipStream_t) {
  const int32_t* starts = *static_cast<int32_t**>(args[0]);
  const int n = *static_cast<int*>(args[1]);
  int32_t* out = *static_cast<int32_t**>(args[4]);
  for (int i = 0; i < n; ++i) out[i] = starts[i] / 2;
  return hipSuccess;
}
hipError_t __hipPushCallConfiguration(dim3, dim3, size_t, hipStream_t) { return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3*, dim3*, size_t*, hipStream_t*) { return hipSuccess; }
void** __hipRegisterFatBinary(const void*) { return nullptr; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
}

namespace sc {
void note_hip_error(int32_t) {}
template <int DT> hipError_t attn_launch(int, const AttnParams&, AttnTiles, int, hipStream_t) { return hipSuccess; }
template <int DT> hipError_t attn_few_launch(int, const AttnParams&, int, hipStream_t) { return hipSuccess; }
template hipError_t attn_launch<kF32>(int, const AttnParams&, AttnTiles, int, hipStream_t);
template hipError_t attn_launch<kF16>(int, const AttnParams&, AttnTiles, int, hipStream_t);
template hipError_t attn_launch<kBF16>(int, const AttnParams&, AttnTiles, int, hipStream_t);
template hipError_t attn_few_launch<kF32>(int, const AttnParams&, int, hipStream_t);
template hipError_t attn_few_launch<kF16>(int, const AttnParams&, int, hipStream_t);
template hipError_t attn_few_launch<kBF16>(int, const AttnParams&, int, hipStream_t);
}  // namespace sc

int main() {
  sizes = new std::map<void*, size_t>;
  const sc_attn_desc desc = {4, 2, 64, SC_BF16, 1, 0, 0.125f};
  const int64_t starts[] = {0, 300, 300, 1000};
  sc_rows set = {};
  set.rows = 1000;
  set.kept = 500;
  set.version = 1;
  size_t bytes = 0;
  if (sparse_attn_workspace_bytes(&desc, 3, 1000, &bytes) != SC_OK) return 1;
  void* workspace = std::aligned_alloc(256, (bytes + 255) / 256 * 256);
  for (fail_at = 1;; ++fail_at) {
    sc_attn* plan = nullptr;
    asked = live = touched = 0;
    n_flying = 0;
    armed = true;
    const sc_status st = sparse_attn_plan(&desc, 3, starts, &set, workspace, bytes, nullptr, &plan);
    if (st == SC_OK) sparse_attn_destroy(plan);
    armed = false;
    std::printf("%ld status %d touched %ld leaked %ld\n", fail_at, (int)st, touched, live);
    if ((st == SC_OK) != (plan != nullptr)) return 2;
    if (asked < fail_at) return st == SC_OK ? 0 : 3;
    if (fail_at > 1000) return 4;
  }
}
