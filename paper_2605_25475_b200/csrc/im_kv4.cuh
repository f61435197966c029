// Format and shared device code of the paged 4-bit KV cache (include/indexmem.h, im_kv4): e2m1 codes in blocks of 16
// channels with an e4m3 scale each.  Code times scale has at most 6 significant bits and lies in [2^-10, 2688], so it is
// exact in f16 and in bf16: the only rounding of the format is the one im_kv4_append makes.
#pragma once
#include <cuda_fp16.h>

#include "im_internal.cuh"

constexpr int KV4_MAX_SEQS = 65535;

// by-value kernel parameter: the cache, sizes in bytes resolved
struct Kv4 {
  uint8_t* pool;
  const int32_t* k_exp;
  const int32_t* v_exp;
  int32_t* status;
  int n_pages, ps, Hkv, d, n_seqs, max_pages;
};

constexpr int kv4_group_bytes(int d) { return 18 * d; }  // 16 tokens, keys and values
__device__ __forceinline__ size_t kv4_group_index(const Kv4& c, int page, int h, int group) {
  return ((size_t)page * c.Hkv + h) * (c.ps >> 4) + group;
}
__device__ __forceinline__ uint8_t* kv4_group(const Kv4& c, int page, int h, int group) {
  return c.pool + kv4_group_index(c, page, h, group) * kv4_group_bytes(c.d);
}
// entry t >= 0 of a sequence: which of its pages, and where in it (page sizes are powers of two; a division is 20 instructions)
__device__ __forceinline__ int kv4_nth_page(const Kv4& c, int t) { return (int)((unsigned)t >> (31 - __clz(c.ps))); }
__device__ __forceinline__ int kv4_slot(const Kv4& c, int t) { return t & (c.ps - 1); }
// offsets inside a group: row r of the key codes / key scales / value codes / value scales
__device__ __forceinline__ int kv4_kc(int d, int r) { return r * (d >> 1); }
__device__ __forceinline__ int kv4_ks(int d, int r) { return 8 * d + r * (d >> 4); }
__device__ __forceinline__ int kv4_vc(int d, int r) { return 9 * d + r * (d >> 1); }
__device__ __forceinline__ int kv4_vs(int d, int r) { return 17 * d + r * (d >> 4); }

// 2^e for the caller's exponents (clamped to the documented range)
__device__ __forceinline__ float kv4_pow2(int e) {
  return __uint_as_float((uint32_t)(127 + max(-60, min(60, e))) << 23);
}
__device__ __forceinline__ int kv4_exp(const int32_t* e, int h) { return e ? max(-60, min(60, e[h])) : 0; }

// the sequence that token t belongs to (the last i with cu[i] <= t, if t < cu[i + 1]), or -1
__device__ __forceinline__ int kv4_find(const int32_t* cu, int n_seqs, int t) {
  if (!cu) return t < n_seqs ? t : -1;
  if (t < cu[0] || t >= cu[n_seqs]) return -1;
  int lo = 0, hi = n_seqs;  // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

// eight e2m1 codes (the low half of a byte first) -> four f16 pairs.  The conversion is only ever applied to the four
// bytes of a whole word: applied to a byte that was loaded as one, nvcc 12.9's code read 0.
__device__ __forceinline__ void kv4_f16_e2m1(uint32_t word, uint32_t* v) {
  asm("{\n\t.reg .b8 a, b, c, e;\n\tmov.b32 {a, b, c, e}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, e;\n\t}"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
      : "r"(word));
}
// two e4m3 scales -> f16 pair
__device__ __forceinline__ uint32_t kv4_f16x2_e4m3(uint32_t two) {
  uint32_t r;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(r) : "r"(two));
  return r;
}
__device__ __forceinline__ float2 kv4_unpack_f16(uint32_t v) {
  return __half22float2(*reinterpret_cast<const __half2*>(&v));
}

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// launch as programmatic dependent of the kernel ahead in the stream: the kernel calls pdl_wait() before it touches
// anything that kernel writes
template <typename... KArgs, typename... Args>
inline cudaError_t kv4_launch(void (*kernel)(KArgs...), dim3 grid, int threads, int smem, cudaStream_t s, bool dependent, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = dependent ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, (KArgs)args...);
}

// host: validates the description (im_kv4.cu); IM_OK and *out, or the error after recording a message that names `fn`
int kv4_describe(const im_kv4* cache, const char* fn, Kv4* out);
int kv4_check_map(const im_kv4_map* m, const char* fn);
int kv4_fail(int code, const char* fn, const char* what);
int kv4_sm_count();  // of the current device (0: none)
size_t kv4_attention_workspace(const Kv4& c, int max_q, int n_q_heads);
inline size_t kv4_align(size_t b) { return (b + 255) & ~(size_t)255; }
