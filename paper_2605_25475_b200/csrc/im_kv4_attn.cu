// Attention over the paged 4-bit KV cache (include/indexmem.h, im_kv4_attention).
#include <math.h>

#include <type_traits>

#include "im_kv4.cuh"

namespace {

constexpr float NEG_INF = -__builtin_huge_valf();

template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<bf16>(bf16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__half* p, float v) { *p = __float2half_rn(v); }

// One block per (query token, query head); the warps take entries in turn, a lane D / 32 channels.
template <int D, typename T, typename OutT>
__global__ void __launch_bounds__(128)
k_kv4_attend(Kv4 c, const int32_t* __restrict__ table, const int32_t* __restrict__ lens, const T* __restrict__ q, long long q_stride,
             const int32_t* __restrict__ cu, int H, float scale, int causal, OutT* __restrict__ out, float* __restrict__ lse) {
  constexpr int CH = D / 32;
  __shared__ float s_acc[4][D];
  __shared__ float s_m[4], s_l[4];
  const int t = blockIdx.x, j = blockIdx.y, h = j / (H / c.Hkv), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int i = kv4_find(cu, c.n_seqs, t);
  if (i < 0) return;
  int L = min(max(lens[i], 0), c.max_pages * c.ps);
  int sees = L;
  if (causal) sees = max(0, min(L, L - (cu ? cu[i + 1] - t : 1) + 1));
  const float ks = scale * kv4_pow2(kv4_exp(c.k_exp, h)), vs = kv4_pow2(kv4_exp(c.v_exp, h));
  float qr[CH], acc[CH];
#pragma unroll
  for (int x = 0; x < CH; ++x) {
    qr[x] = to_float<T>(q[t * q_stride + (size_t)j * D + lane * CH + x]);
    acc[x] = 0.f;
  }
  float m = NEG_INF, l = 0.f;
  for (int e = warp; e < sees; e += 4) {
    const int page = table[(size_t)i * c.max_pages + e / c.ps], r = e & 15;
    if (page < 0 || page >= c.n_pages) {
      if (lane == 0) atomicOr(c.status, IM_KV4_BAD_MAP);
      continue;
    }
    const uint8_t* g = kv4_group(c, page, h, e % c.ps >> 4);
    float s = 0.f, v[CH];
    const float sk = kv4_unpack_f16(kv4_f16x2_e4m3(g[kv4_ks(D, r) + lane * CH / 16])).x;
    const float sv = kv4_unpack_f16(kv4_f16x2_e4m3(g[kv4_vs(D, r) + lane * CH / 16])).x;
    uint32_t kw[4], vw[4];  // the eight channels of the word that holds the lane's
    kv4_f16_e2m1(*reinterpret_cast<const uint32_t*>(g + kv4_kc(D, r) + (lane * CH / 8) * 4), kw);
    kv4_f16_e2m1(*reinterpret_cast<const uint32_t*>(g + kv4_vc(D, r) + (lane * CH / 8) * 4), vw);
#pragma unroll
    for (int x = 0; x < CH; x += 2) {
      const int at = (lane * CH + x) / 2 % 4;
      const float2 a = kv4_unpack_f16(at == 0 ? kw[0] : at == 1 ? kw[1] : at == 2 ? kw[2] : kw[3]);
      const float2 b = kv4_unpack_f16(at == 0 ? vw[0] : at == 1 ? vw[1] : at == 2 ? vw[2] : vw[3]);
      s = fmaf(qr[x], a.x * sk, fmaf(qr[x + 1], a.y * sk, s));
      v[x] = b.x * sv;
      v[x + 1] = b.y * sv;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    s *= ks;
    const float mn = fmaxf(m, s), corr = expf(m - mn), p = expf(s - mn);
    l = l * corr + p;
#pragma unroll
    for (int x = 0; x < CH; ++x) acc[x] = fmaf(p, v[x], acc[x] * corr);
    m = mn;
  }
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
#pragma unroll
  for (int x = 0; x < CH; ++x) s_acc[warp][lane * CH + x] = acc[x];
  __syncthreads();
  float M = NEG_INF, total = 0.f;
  for (int w = 0; w < 4; ++w) M = fmaxf(M, s_m[w]);
  float f[4];
  for (int w = 0; w < 4; ++w) {
    f[w] = s_m[w] > NEG_INF ? expf(s_m[w] - M) : 0.f;
    total = fmaf(s_l[w], f[w], total);
  }
  for (int x = threadIdx.x; x < D; x += 128) {
    float o = 0.f;
    for (int w = 0; w < 4; ++w) o = fmaf(s_acc[w][x], f[w], o);
    put(out + ((size_t)t * H + j) * D + x, total == 0.f ? 0.f : o / total * vs);
  }
  if (lse && threadIdx.x == 0) lse[(size_t)t * H + j] = total == 0.f ? NEG_INF : M + logf(total);
}

template <int D, typename T>
cudaError_t launch(const Kv4& c, const im_kv4_map* m, const void* q, long long q_stride, int n_tokens, const int32_t* cu, int H, float scale,
                   int causal, void* out, int out_f32, float* lse, cudaStream_t s) {
  const dim3 grid(n_tokens, H);
  if (out_f32) k_kv4_attend<D, T, float><<<grid, 128, 0, s>>>(c, m->table, m->lens, (const T*)q, q_stride, cu, H, scale, causal, (float*)out, lse);
  else k_kv4_attend<D, T, T><<<grid, 128, 0, s>>>(c, m->table, m->lens, (const T*)q, q_stride, cu, H, scale, causal, (T*)out, lse);
  return cudaGetLastError();
}

}  // namespace

size_t kv4_attention_workspace(const Kv4& c, int n_tokens, int n_q_heads) { return 256; }

extern "C" int im_kv4_attention(const im_kv4* cache, const im_kv4_map* map, int dtype, const void* q, long long q_stride, int n_tokens,
                                const int32_t* cu_q, int max_q, int n_q_heads, float softmax_scale, int causal, void* out, int out_f32,
                                float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const char* fn = "im_kv4_attention";
  Kv4 c;
  int rc = kv4_describe(cache, fn, &c);
  if (rc == IM_OK) rc = kv4_check_map(map, fn);
  if (rc != IM_OK) return rc;
  if (dtype != IM_BF16 && dtype != IM_F16) return kv4_fail(IM_ERR_ARG, fn, "queries are bf16 or f16");
  if (n_q_heads < 1 || n_q_heads % c.Hkv || n_q_heads > 65535) return kv4_fail(IM_ERR_ARG, fn, "n_q_heads must be a multiple of n_kv_heads");
  if (n_tokens < 0 || max_q < 0 || (!cu_q && n_tokens != c.n_seqs)) return kv4_fail(IM_ERR_ARG, fn, "bad token count");
  if (n_tokens && (!q || !out)) return kv4_fail(IM_ERR_ARG, fn, "null tensor");
  const long long dense = (long long)n_q_heads * c.d;
  if (!q_stride) q_stride = dense;
  if (q_stride < dense || q_stride % 8 || (((uintptr_t)q | (uintptr_t)out) & 15) || ((uintptr_t)lse & 3))
    return kv4_fail(IM_ERR_ARG, fn, "the token stride must be a multiple of 8 elements, no shorter than a token; bases 16-byte aligned");
  if (!(softmax_scale >= 0.f) || isinf(softmax_scale)) return kv4_fail(IM_ERR_ARG, fn, "softmax_scale must be positive (0: 1/sqrt(head_dim))");
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < kv4_attention_workspace(c, n_tokens, n_q_heads))
    return kv4_fail(IM_ERR_CAPACITY, fn, "workspace missing, misaligned or too small");
  if (!n_tokens) return IM_OK;
  const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)c.d);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  auto go = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    return dtype == IM_BF16 ? launch<D, bf16>(c, map, q, q_stride, n_tokens, cu_q, n_q_heads, scale, causal, out, out_f32, lse, s)
                            : launch<D, __half>(c, map, q, q_stride, n_tokens, cu_q, n_q_heads, scale, causal, out, out_f32, lse, s);
  };
  const cudaError_t e = c.d == 64    ? go(std::integral_constant<int, 64>{})
                        : c.d == 128 ? go(std::integral_constant<int, 128>{})
                                     : go(std::integral_constant<int, 256>{});
  return e == cudaSuccess ? IM_OK : im_fail_message(IM_ERR_CUDA, cudaGetErrorString(e));
}
