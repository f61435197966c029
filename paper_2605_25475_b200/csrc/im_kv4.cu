// The paged 4-bit KV cache's calls other than attention: append (plan + store), gather, fork, compact (scan + plan +
// move).  See include/indexmem.h for the contract and the format.
//
// All of them move bytes.  The integer part (which page goes where) is one launch of one CTA, or of eight that share their
// counts through distributed shared memory: the answer has to be the same whatever order the hardware runs things in, so
// pages are ranked by prefix sums and nothing depends on the order of atomics.
#include <cooperative_groups.h>
#include <stdio.h>

#include "im_kv4.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int PLAN_CTAS = 8, PLAN_THREADS = 1024, PLAN_SEG = 128, PLAN_WARPS = PLAN_THREADS / 32;
constexpr int SCAN_THREADS = 1024;
constexpr int PLAN_ONE_CTA_PAGES = 8192;
enum { PLAN_APPEND = 0, PLAN_COMPACT = 1 };

// What a plan hands to the kernels behind it (in the caller's workspace; every word that is read is written by the same call).
struct PlanWs {
  int32_t* ok;    // [1] 1: the call is made, 0: nothing changes
  int32_t* len;   // [n_seqs] lengths before the call
  int32_t* off;   // [n_seqs] rank of the sequence's first new page
  int32_t* info;  // [n_seqs] append: the shared last page whose tokens are copied, or -1; compact: pages that stay
  int32_t* cnt;   // [n_seqs] compact: survivors, or -1 for a row that is out of order
  int32_t* list;  // [list_max] the free pages in ascending order
  int32_t* goff;  // [n_seqs + 1] compact: groups of 16 survivors to move, ahead of the sequence
  int32_t* src;   // [n_seqs][cap] compact: page * page_size + slot of the survivors
  int list_max, cap;
};

template <typename N>
__device__ __forceinline__ N warp_scan_incl(N v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const N u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}
// exclusive scan over the block; *total receives the block's sum
template <int WARPS, typename N>
__device__ __forceinline__ N block_scan(N v, N* s_warp, N* total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const N incl = warp_scan_incl(v, lane);
  __syncthreads();  // (the previous scan's readers are through with s_warp)
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    const N w = warp_scan_incl(lane < WARPS ? s_warp[lane] : (N)0, lane);
    if (lane < WARPS) s_warp[lane] = w;
  }
  __syncthreads();
  *total = s_warp[WARPS - 1];
  return incl - v + (warp ? s_warp[warp - 1] : 0);
}

// [lo, hi) of the tokens of sequence i; ok = 0 if cu is out of order
__device__ __forceinline__ int new_tokens(const int32_t* cu, int i, int n_tokens, bool* bad) {
  if (!cu) return 1;
  const int a = cu[i], b = cu[i + 1];
  if (a < 0 || b < a || b > n_tokens) {
    *bad = true;
    return 0;
  }
  return b - a;
}

// Gives out pages.  One cluster; the sequences' needs are added up by every CTA for itself (they are few), the free pages
// are counted and listed by shares.  Phases are separated by cluster barriers, so that with from == to nothing is written
// before everybody has read what the decision depends on.  Bound by its chain of round trips (lengths, free pages, list,
// rows): 9 to 12 us alone, for 32 sequences on 2,100 pages, 16 on 4,100.
template <int MODE>
__global__ void __launch_bounds__(PLAN_THREADS)
k_kv4_plan(Kv4 c, im_kv4_map from, im_kv4_map to, const int32_t* __restrict__ cu, int n_tokens, PlanWs ws) {
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ long long s_warp[PLAN_WARPS];
  __shared__ int s_free[PLAN_WARPS];
  __shared__ int s_count;
  const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks(), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_release();
  if (MODE == PLAN_COMPACT) pdl_wait();  // (the scan kernel's counts)
  // ---- what each sequence needs
  long long total = 0, moves = 0;
  bool bad = false, full = false;
  for (int base = 0; base < c.n_seqs; base += PLAN_THREADS) {
    const int i = base + tid;
    int need = 0, move = 0, info = MODE == PLAN_APPEND ? -1 : 0, L = 0;
    if (i < c.n_seqs) {
      L = from.lens[i];
      if (MODE == PLAN_APPEND) {
        const int add = new_tokens(cu, i, n_tokens, &bad);
        if (L < 0 || L > c.max_pages * c.ps) {
          bad = true;
        } else if (L + (long long)add > (long long)c.max_pages * c.ps) {
          full = true;
        } else {
          need = (L + add + c.ps - 1) / c.ps - (L + c.ps - 1) / c.ps;
          if (add > 0 && L % c.ps) {
            const int last = from.table[(size_t)i * c.max_pages + L / c.ps];
            if (last < 0 || last >= c.n_pages) bad = true;
            else if (from.refs[last] > 1) {
              info = last;
              ++need;
            }
          }
        }
      } else {
        const int cnt = ws.cnt[i];
        if (cnt < 0) bad = true;
        else {
          need = (cnt + c.ps - 1) / c.ps - ws.info[i];
          move = max(0, (cnt - ws.info[i] * c.ps + 15) >> 4);
        }
      }
    }
    long long chunk;
    const long long before = block_scan<PLAN_WARPS>((long long)need, s_warp, &chunk);
    if (rank == 0 && i < c.n_seqs) {
      const long long o = total + before;
      ws.len[i] = L;
      ws.off[i] = (int)(o < 0x7fffffff ? o : 0x7fffffff);
      if (MODE == PLAN_APPEND) ws.info[i] = info;
    }
    total += chunk;
    if (MODE == PLAN_COMPACT) {
      const long long ahead = block_scan<PLAN_WARPS>((long long)move, s_warp, &chunk);
      if (rank == 0 && i < c.n_seqs) ws.goff[i] = (int)(moves + ahead);
      moves += chunk;
    }
  }
  if (MODE == PLAN_COMPACT && rank == 0 && tid == 0) ws.goff[c.n_seqs] = (int)moves;
  bad = __syncthreads_or(bad);
  full = __syncthreads_or(full);
  // ---- free pages of this CTA's share, in runs per warp
  const int share = (c.n_pages + ctas - 1) / ctas;
  const int p0 = min(c.n_pages, rank * share), p1 = min(c.n_pages, p0 + share);
  const int run = ((p1 - p0 + PLAN_WARPS - 1) / PLAN_WARPS + 31) & ~31;
  const int w0 = min(p1, p0 + warp * run), w1 = min(p1, w0 + run);
  const bool want = total > 0 && !bad && !full;  // the same in every CTA
  if (want) {
    int n = 0;
#pragma unroll 4
    for (int p = w0; p < w1; p += 32)
      n += __popc(__ballot_sync(0xffffffffu, p + lane < w1 && from.refs[p + lane] == 0));
    if (lane == 0) s_free[warp] = n;
  }
  __syncthreads();
  if (warp == 0) {
    const int k = want ? s_free[lane] : 0, incl = warp_scan_incl(k, lane);
    s_free[lane] = incl - k;
    if (lane == 31) s_count = incl;
  }
  __syncthreads();
  cluster.sync();
  int first = 0, free_pages = 0;
  if (want)
    for (int r = 0; r < ctas; ++r) {
      const int n = *cluster.map_shared_rank(&s_count, r);
      if (r < rank) first += n;
      free_pages += n;
    }
  const bool ok = !bad && !full && (total == 0 || total <= free_pages);
  if (rank == 0 && tid == 0) {
    *ws.ok = ok ? 1 : 0;
    const int bits = (bad ? IM_KV4_BAD_MAP : 0) | (!bad && !ok ? IM_KV4_NO_PAGES : 0);
    if (bits) atomicOr(c.status, bits);
  }
  // ---- list them, and count the new holders
  const bool copy_refs = to.refs != from.refs;
  if ((want && ok) || copy_refs) {
    int at = first + (want ? s_free[warp] : 0);
    for (int p = w0; p < w1 && (copy_refs || at < total); p += 32) {
      const int r = p + lane < w1 ? from.refs[p + lane] : 1;
      const bool hit = want && ok && r == 0;
      const unsigned m = __ballot_sync(0xffffffffu, hit);
      const int nth = at + __popc(m & ((1u << lane) - 1u));
      const bool taken = hit && nth < total;
      if (taken) ws.list[nth] = p + lane;
      if (p + lane < w1 && (taken || copy_refs)) to.refs[p + lane] = taken ? 1 : r;
      at += __popc(m);
    }
  }
  cluster.sync();  // (also the last read of another CTA's shared memory)
  // ---- rows, in pieces of PLAN_SEG entries
  const int segs = (c.max_pages + PLAN_SEG - 1) / PLAN_SEG;
  for (long long task = rank * PLAN_WARPS + warp; task < (long long)c.n_seqs * segs; task += ctas * PLAN_WARPS) {
    const int i = (int)(task / segs), j0 = (int)(task % segs) * PLAN_SEG;
    const int L = ws.len[i], off = ws.off[i], info = ws.info[i];
    const size_t row = (size_t)i * c.max_pages;
    const int held = L < 0 ? 0 : (int)min((long long)c.max_pages, ((long long)L + c.ps - 1) / c.ps);
    int kept = held, pages = held, len = L;
    if (ok) {
      if (MODE == PLAN_APPEND) {
        bool b = false;
        len = L + new_tokens(cu, i, n_tokens, &b);
        pages = (len + c.ps - 1) / c.ps;
        if (info >= 0) kept = held - 1;
      } else {
        len = ws.cnt[i];
        pages = (len + c.ps - 1) / c.ps;
        kept = info;
      }
    }
    int old[PLAN_SEG / 32], now[PLAN_SEG / 32];
#pragma unroll
    for (int q = 0; q < PLAN_SEG / 32; ++q) {
      const int j = j0 + 32 * q + lane;
      old[q] = j < held ? from.table[row + j] : -1;
      now[q] = j < kept || j >= pages ? old[q] : ws.list[off + j - kept];
    }
#pragma unroll
    for (int q = 0; q < PLAN_SEG / 32; ++q) {
      const int j = j0 + 32 * q + lane;
      if (ok && j >= kept && j < held && old[q] >= 0 && old[q] < c.n_pages) atomicSub(to.refs + old[q], 1);
      if (j < pages) to.table[row + j] = now[q];
    }
    if (j0 == 0 && lane == 0) to.lens[i] = len;
  }
}

// ------------------------------------------------------------------ append: quantise and store
// One block of 16 values -> 8 code bytes and a scale.  x has at most 11 significant bits (bf16 or f16 input times a
// power of two) and a code edge times the scale at most 7, so a quotient that is not exactly on an edge is 2^-11 (relative) away
// from it: amax / 6 in float32 decides the scale exactly, and x * (1 / scale), off by 2 ulp, decides the code exactly
// once it is snapped to multiples of 2^-15 (adding and subtracting 384), which puts ties back on their edge.  Quotients above 128
// are snapped more coarsely, and are far beyond the last edge all the same: the conversion takes them to 6.
__device__ __forceinline__ uint2 quantise16(const float* x, uint8_t* scale) {
  float amax = 0.f;
#pragma unroll
  for (int k = 0; k < 16; k += 2)
    asm("{\n\t.reg .f32 a, b;\n\tabs.f32 a, %1;\n\tabs.f32 b, %2;\n\tmax.f32 %0, %0, a, b;\n\t}" : "+f"(amax) : "f"(x[k]), "f"(x[k + 1]));
  uint32_t s8;
  asm("{\n\t.reg .b16 t;\n\tcvt.rn.satfinite.e4m3x2.f32 t, %2, %1;\n\tcvt.u32.u16 %0, t;\n\t}" : "=r"(s8) : "f"(__fdiv_rn(amax, 6.0f)), "f"(0.f));
  *scale = (uint8_t)s8;
  const float s = kv4_unpack_f16(kv4_f16x2_e4m3(s8)).x;
  const float inv = s > 0.f ? __frcp_rn(s) : 0.f;
  uint32_t w[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float v = x[8 * q + k];
      const float m = __fadd_rn(__fadd_rn(__fmul_rn(fabsf(v), inv), 384.0f), -384.0f);
      y[k] = copysignf(m, v);
    }
    asm("{\n\t.reg .b8 a, b, c, e;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 e, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, e};\n\t}"
        : "=r"(w[q])
        : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  }
  return make_uint2(w[0], w[1]);
}

template <typename T>
__device__ __forceinline__ float2 two_floats(uint32_t v);
template <>
__device__ __forceinline__ float2 two_floats<bf16>(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 two_floats<__half>(uint32_t v) {
  return kv4_unpack_f16(v);
}

// One thread per block of 16 channels, keys and values; grid.y = head, grid.x over (token, block): a warp reads whole rows and
// writes the code rows of neighbouring tokens of one head, which lie side by side.  The rows of the grid behind those copy
// the tokens of shared last pages.  The loads run ahead of the wait for the plan, and the lookups in its map (two round
// trips) ahead of the quantiser.  Bound by the ALU pipe (70 % of it before finiteness went to one multiply-add per value, and the
// maximum to three operands, 81.5 -> 75.1 us): 24,456 f16 tokens of 8 heads of 128, the append and its reading back, 70 us.
constexpr int STORE_THREADS = 256;
template <typename T>
__global__ void __launch_bounds__(STORE_THREADS)
k_kv4_store(Kv4 c, const int32_t* __restrict__ table, const int32_t* __restrict__ lens, const T* __restrict__ k, long long k_stride,
            const T* __restrict__ v, long long v_stride, int n_tokens, const int32_t* __restrict__ cu, PlanWs ws) {
  const int h = blockIdx.y;
  if (h >= c.Hkv) {  // (sequence, head) by (sequence, head)
    const int cow = (blockIdx.y - c.Hkv) * gridDim.x + blockIdx.x, step = (gridDim.y - c.Hkv) * gridDim.x;
    pdl_wait();
    if (!*ws.ok) return;
    for (int task = cow; task < c.n_seqs * c.Hkv; task += step) {
      const int i = task / c.Hkv, hh = task % c.Hkv;
      const int old = ws.info[i];
      if (old < 0) continue;
      const int L = lens[i] - (cu ? cu[i + 1] - cu[i] : 1), rows = L % c.ps;
      const int fresh = table[(size_t)i * c.max_pages + L / c.ps];
      const uint8_t* a = kv4_group(c, old, hh, 0);
      uint8_t* b = kv4_group(c, fresh, hh, 0);
      const int row16 = c.d >> 5, group = kv4_group_bytes(c.d);  // 16-byte pieces of a code row
      // the rows of a section lie side by side: whole pieces of the codes, words of the scales
#pragma unroll 2
      for (int e = threadIdx.x; e < rows * 2 * row16; e += STORE_THREADS) {
        const int r = e / (2 * row16), x = e % (2 * row16);
        const int o = (r >> 4) * group + (x < row16 ? kv4_kc(c.d, r & 15) + 16 * x : kv4_vc(c.d, r & 15) + 16 * (x - row16));
        *reinterpret_cast<uint4*>(b + o) = *reinterpret_cast<const uint4*>(a + o);
      }
      const int row4 = c.d >> 6;
      for (int e = threadIdx.x; e < rows * 2 * row4; e += STORE_THREADS) {
        const int r = e / (2 * row4), x = e % (2 * row4);
        const int o = (r >> 4) * group + (x < row4 ? kv4_ks(c.d, r & 15) + 4 * x : kv4_vs(c.d, r & 15) + 4 * (x - row4));
        *reinterpret_cast<uint32_t*>(b + o) = *reinterpret_cast<const uint32_t*>(a + o);
      }
    }
    return;
  }
  const int lg = c.d == 64 ? 2 : c.d == 128 ? 3 : 4;  // log2 of the blocks of a row
  const int idx = blockIdx.x * STORE_THREADS + threadIdx.x, blk = idx & ((1 << lg) - 1), t = idx >> lg;
  uint4 in[4] = {};
  int i = -1;
  if (t < n_tokens) {
    const uint4* ks = reinterpret_cast<const uint4*>(k + t * k_stride + (size_t)h * c.d + blk * 16);
    const uint4* vs = reinterpret_cast<const uint4*>(v + t * v_stride + (size_t)h * c.d + blk * 16);
    in[0] = ks[0], in[1] = ks[1], in[2] = vs[0], in[3] = vs[1];
    i = kv4_find(cu, c.n_seqs, t);
  }
  pdl_wait();
  if (i < 0) return;
  const int ok = *ws.ok, slot = lens[i] - (cu ? cu[i + 1] - t : 1);
  const int nth = slot >= 0 ? kv4_nth_page(c, slot) : c.max_pages;
  const int page = ok && nth < c.max_pages ? table[(size_t)i * c.max_pages + nth] : -1;
  bool odd = false;
  uint2 codes[2];
  uint8_t scale[2];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const uint4 a = in[2 * which], b = in[2 * which + 1];
    const uint32_t raw[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    const float down = kv4_pow2(-kv4_exp(which ? c.v_exp : c.k_exp, h));
    float x[16], none = 0.f;  // none: 0 times everything, which is NaN if anything is not finite
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float2 f = two_floats<T>(raw[q]);
      none = fmaf(f.x, 0.f, fmaf(f.y, 0.f, none));
      x[2 * q] = f.x * down;
      x[2 * q + 1] = f.y * down;
    }
    if (none != 0.f) {
      odd = true;
#pragma unroll
      for (int k = 0; k < 16; ++k) x[k] = x[k] == x[k] ? x[k] : 0.f;
    }
    codes[which] = quantise16(x, &scale[which]);
  }
  if (odd) atomicOr(c.status, IM_KV4_NONFINITE);
  if (page < 0 || page >= c.n_pages) return;  // (the call is not made, as the plan has flagged)
  const int at = kv4_slot(c, slot);
  uint8_t* g = kv4_group(c, page, h, at >> 4);
  *reinterpret_cast<uint2*>(g + kv4_kc(c.d, at & 15) + 8 * blk) = codes[0];
  g[kv4_ks(c.d, at & 15) + blk] = scale[0];
  *reinterpret_cast<uint2*>(g + kv4_vc(c.d, at & 15) + 8 * blk) = codes[1];
  g[kv4_vs(c.d, at & 15) + blk] = scale[1];
}

// ------------------------------------------------------------------ gather
// One thread per (row, head, 8 channels), keys and values: index in the order of the output, which is what most of the
// bytes are, so that a warp writes 512 bytes side by side.  Bound by issue slots (79 % busy
// before the divisions by the page size became shifts).  131,072 rows of 8 heads of 128: 155 us to bf16 (4.4 TB/s, 68 % of a copy),
// 265 us to float32 (4.6 TB/s, 70 %).
constexpr int GATHER_THREADS = 256;
template <typename T>
__device__ __forceinline__ uint32_t pack_two(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack_two<bf16>(float a, float b) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
template <>
__device__ __forceinline__ uint32_t pack_two<__half>(float a, float b) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
template <typename T>
__device__ __forceinline__ void put8(T* dst, uint32_t codes, uint8_t scale, float up) {
  uint32_t pair[4];
  kv4_f16_e2m1(codes, pair);
  const float s = kv4_unpack_f16(kv4_f16x2_e4m3(scale)).x * up;
  float2 f[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f[q] = kv4_unpack_f16(pair[q]);
    f[q].x *= s;
    f[q].y *= s;
  }
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(dst)[0] = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
    reinterpret_cast<float4*>(dst)[1] = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
  } else {
    *reinterpret_cast<uint4*>(dst) =
        make_uint4(pack_two<T>(f[0].x, f[0].y), pack_two<T>(f[1].x, f[1].y), pack_two<T>(f[2].x, f[2].y), pack_two<T>(f[3].x, f[3].y));
  }
}

template <typename T>
__global__ void __launch_bounds__(GATHER_THREADS)
k_kv4_gather(Kv4 c, const int32_t* __restrict__ table, const int32_t* __restrict__ lens, int n_rows, const int32_t* __restrict__ cu,
             const int32_t* __restrict__ slots, T* __restrict__ k, T* __restrict__ v) {
  const int lg = c.d == 64 ? 3 : c.d == 128 ? 4 : 5;  // log2 of the threads of a row
  const unsigned idx = blockIdx.x * GATHER_THREADS + threadIdx.x;
  const int x = (int)(idx & ((1u << lg) - 1u));
  const unsigned rh = idx >> lg;
  const int r = (int)(rh / (unsigned)c.Hkv), h = (int)(rh % (unsigned)c.Hkv);
  if (r >= n_rows) return;
  int slot = slots ? slots[r] : 0;
  const int i = kv4_find(cu, c.n_seqs, r);
  if (i < 0) return;
  if (!slots && cu) slot = r - cu[i];
  uint32_t kc = 0, vc = 0;
  uint8_t ks = 0, vs = 0;
  if (slot >= 0 && slot < lens[i] && kv4_nth_page(c, slot) < c.max_pages) {
    const int page = table[(size_t)i * c.max_pages + kv4_nth_page(c, slot)];
    if (page >= 0 && page < c.n_pages) {
      const int at = kv4_slot(c, slot);
      const uint8_t* g = kv4_group(c, page, h, at >> 4);
      kc = *reinterpret_cast<const uint32_t*>(g + kv4_kc(c.d, at & 15) + 4 * x);
      ks = g[kv4_ks(c.d, at & 15) + (x >> 1)];
      vc = *reinterpret_cast<const uint32_t*>(g + kv4_vc(c.d, at & 15) + 4 * x);
      vs = g[kv4_vs(c.d, at & 15) + (x >> 1)];
    } else if (x == 0) {
      atomicOr(c.status, IM_KV4_BAD_MAP);
    }
  }
  const size_t at = (size_t)idx * 8;
  if (k) put8(k + at, kc, ks, kv4_pow2(kv4_exp(c.k_exp, h)));
  if (v) put8(v + at, vc, vs, kv4_pow2(kv4_exp(c.v_exp, h)));
}

// ------------------------------------------------------------------ fork
// refs of `to` start as those of `from`; then every row adds one to the pages of its new row and takes one off those of
// its old row.  Integer sums: the order does not matter.  Bound by its launches: 4.7 us for 1024 rows and refs apart.
__global__ void k_kv4_copy_refs(const int32_t* __restrict__ a, int32_t* __restrict__ b, int n) {
  pdl_release();
  for (int p = blockIdx.x * blockDim.x + threadIdx.x; p < n; p += gridDim.x * blockDim.x) b[p] = a[p];
}

constexpr int FORK_THREADS = 256, FORK_SEG = 128;  // a warp handles 128 entries of a row
__global__ void __launch_bounds__(FORK_THREADS)
k_kv4_fork(Kv4 c, im_kv4_map from, im_kv4_map to, const int32_t* __restrict__ parent, int segs) {
  const long long w = ((long long)blockIdx.x * FORK_THREADS + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31, i = (int)(w / segs), j0 = (int)(w % segs) * FORK_SEG;
  if (i >= c.n_seqs) return;  // (a block that ends counts as having waited)
  int p = parent[i];
  bool bad = false;
  if (p < -1 || p >= c.n_seqs) {
    bad = true;
    p = i;
  }
  const int L = from.lens[i], Lp = p < 0 ? 0 : from.lens[p];
  const long long top = (long long)c.max_pages * c.ps;
  bad |= L < 0 || L > top || Lp < 0 || Lp > top;
  const int held = (int)((min(max((long long)L, 0ll), top) + c.ps - 1) / c.ps);
  const int pages = (int)((min(max((long long)Lp, 0ll), top) + c.ps - 1) / c.ps);
  int mine[FORK_SEG / 32], old[FORK_SEG / 32];
#pragma unroll
  for (int q = 0; q < FORK_SEG / 32; ++q) {
    const int j = j0 + 32 * q + lane;
    mine[q] = j < pages ? from.table[(size_t)p * c.max_pages + j] : -1;
    old[q] = j < held ? from.table[(size_t)i * c.max_pages + j] : -1;
  }
  pdl_wait();
#pragma unroll
  for (int q = 0; q < FORK_SEG / 32; ++q) {
    const int j = j0 + 32 * q + lane;
    if (j < pages) {
      to.table[(size_t)i * c.max_pages + j] = mine[q];
      if (mine[q] < 0 || mine[q] >= c.n_pages) bad = true;
    }
    if (p != i) {
      if (j < pages && mine[q] >= 0 && mine[q] < c.n_pages) atomicAdd(to.refs + mine[q], 1);
      if (j < held && old[q] >= 0 && old[q] < c.n_pages) atomicSub(to.refs + old[q], 1);
    }
  }
  if (bad) atomicOr(c.status, IM_KV4_BAD_MAP);
  if (j0 == 0 && lane == 0) to.lens[i] = Lp;
}

// ------------------------------------------------------------------ compact
// Survivors of one sequence: their rows in the pool, in order, and the pages ahead of the first hole.  One block per
// sequence, 16 flags per thread and round.  6 us for 2176 entries a sequence, 10 us for 32768: round trips.
__global__ void __launch_bounds__(SCAN_THREADS)
k_kv4_scan(Kv4 c, im_kv4_map from, const uint8_t* __restrict__ keep, int keep_stride, PlanWs ws) {
  __shared__ int s_warp[SCAN_THREADS / 32];
  __shared__ int s_hole;
  pdl_release();
  const int i = blockIdx.x, tid = threadIdx.x;
  const int L = from.lens[i];
  if (L < 0 || L > keep_stride || L > (long long)c.max_pages * c.ps) {
    if (tid == 0) {
      ws.cnt[i] = -1;
      ws.info[i] = 0;
    }
    return;
  }
  const uint8_t* row = keep + (size_t)i * keep_stride;
  const bool wide = ((uintptr_t)row & 15) == 0;
  const int32_t* table = from.table + (size_t)i * c.max_pages;
  if (tid == 0) s_hole = L;
  int done = 0, hole = L;
  bool bad = false;
  for (int base = 0; base < L; base += SCAN_THREADS * 16) {
    const int t0 = base + tid * 16;
    uint32_t flags = 0;  // bit k: entry t0 + k survives
    if (t0 < L) {
      if (wide && t0 + 16 <= L) {
        const uint4 v = *reinterpret_cast<const uint4*>(row + t0);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 16; ++k) flags |= ((w[k >> 2] >> (8 * (k & 3))) & 0xffu) ? 1u << k : 0u;
      } else {
        for (int k = 0; k < 16 && t0 + k < L; ++k) flags |= row[t0 + k] ? 1u << k : 0u;
      }
      const uint32_t all = L - t0 >= 16 ? 0xffffu : (1u << (L - t0)) - 1u;
      if (flags != all && hole == L) hole = t0 + __ffs(~flags & all) - 1;
    }
    int chunk;
    int at = done + block_scan<SCAN_THREADS / 32>(__popc(flags), s_warp, &chunk);
    if (flags) {  // 16 entries starting at a multiple of 16 lie in one page
      const int page = table[kv4_nth_page(c, t0)];
      if (page < 0 || page >= c.n_pages) bad = true;
      const int r0 = page * c.ps + kv4_slot(c, t0);
      for (uint32_t m = flags; m; m &= m - 1) ws.src[(size_t)i * ws.cap + at++] = r0 + __ffs(m) - 1;
    }
    done += chunk;
  }
  bad = __syncthreads_or(bad);
  if (hole < L) atomicMin(&s_hole, hole);
  __syncthreads();
  if (tid == 0) {
    ws.cnt[i] = bad ? -1 : done;
    ws.info[i] = s_hole == L ? (L + c.ps - 1) / c.ps : s_hole / c.ps;
  }
}

// A warp writes one group of 16 tokens of one head (18 d bytes side by side) from wherever its tokens were.  Every block has an equal
// run of the groups to move, whatever the sequences are; the warps take the heads, and while a group moves the
// places of the next one's tokens are fetched.  One entry in four of 392,381 surviving, 8 heads of 128: 69 us, 302 MB of entries
// (4.4 TB/s) and 387 MB of DRAM traffic (5.4 TB/s, 82 % of a copy), since a scale row of 8 bytes is read in sectors of 32.
// Held to 40 registers, for half as many more warps, it spilled: the whole call took 102 us instead of 95.
constexpr int MOVE_THREADS = 256;
template <int D>
__global__ void __launch_bounds__(MOVE_THREADS) k_kv4_move(Kv4 c, const int32_t* __restrict__ table, PlanWs ws) {
  constexpr int ROW16 = D / 32;            // 16-byte pieces of a code row
  constexpr int CODES = 2 * 16 * ROW16;    // of a group: keys, then values
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  const int total = ws.goff[c.n_seqs];
  if (!*ws.ok || !total) return;
  const int t0 = (int)((long long)total * blockIdx.x / gridDim.x), t1 = (int)((long long)total * (blockIdx.x + 1) / gridDim.x);
  if (t0 >= t1) return;
  int i = 0;
  for (int hi = c.n_seqs; hi - i > 1;) {  // goff[i] <= t0 < goff[hi]
    const int mid = (i + hi) >> 1;
    if (ws.goff[mid] <= t0) i = mid;
    else hi = mid;
  }
  while (ws.goff[i + 1] <= t0) ++i;
  // group t: rows of it, its page, and (lane r) where row r % 16 was
  struct Group {
    int rows, page, slot, src;
  };
  auto fetch = [&](int t) {
    while (ws.goff[i + 1] <= t) ++i;
    Group g;
    const int j0 = ws.info[i] * c.ps + (t - ws.goff[i]) * 16;
    g.rows = min(16, ws.cnt[i] - j0);
    g.slot = kv4_slot(c, j0);
    g.page = table[(size_t)i * c.max_pages + kv4_nth_page(c, j0)];
    g.src = (lane & 15) < g.rows ? ws.src[(size_t)i * ws.cap + j0 + (lane & 15)] : 0;
    return g;
  };
  Group next = fetch(t0);
  for (int t = t0; t < t1; ++t) {
    const Group now = next;
    if (t + 1 < t1) next = fetch(t + 1);
    const int from = (lane & 15) < now.rows ? now.src : 0;
    for (int h = warp; h < c.Hkv; h += MOVE_THREADS / 32) {
      uint8_t* g = kv4_group(c, now.page, h, now.slot >> 4);
      uint4 code[CODES / 32];
#pragma unroll
      for (int q = 0; q < CODES / 32; ++q) {
        const int e = q * 32 + lane, which = e / (16 * ROW16), r = e / ROW16 % 16, x = e % ROW16;
        const int s = __shfl_sync(0xffffffffu, from, r);
        const uint8_t* a = kv4_group(c, kv4_nth_page(c, s), h, kv4_slot(c, s) >> 4) + (which ? kv4_vc(D, s & 15) : kv4_kc(D, s & 15)) + 16 * x;
        code[q] = r < now.rows ? *reinterpret_cast<const uint4*>(a) : make_uint4(0u, 0u, 0u, 0u);
      }
      // scales: lane = (which, row), D / 16 bytes each
      const int which = lane >> 4, r = lane & 15;
      const uint8_t* a = kv4_group(c, kv4_nth_page(c, from), h, kv4_slot(c, from) >> 4) + (which ? kv4_vs(D, from & 15) : kv4_ks(D, from & 15));
      uint32_t scale[D / 64];
#pragma unroll
      for (int q = 0; q < D / 64; ++q) scale[q] = r < now.rows ? reinterpret_cast<const uint32_t*>(a)[q] : 0u;
#pragma unroll
      for (int q = 0; q < CODES / 32; ++q) {
        const int e = q * 32 + lane, wh = e / (16 * ROW16), rr = e / ROW16 % 16, x = e % ROW16;
        if (rr < now.rows) *reinterpret_cast<uint4*>(g + (wh ? kv4_vc(D, rr) : kv4_kc(D, rr)) + 16 * x) = code[q];
      }
      if (r < now.rows) {
        uint32_t* b = reinterpret_cast<uint32_t*>(g + (which ? kv4_vs(D, r) : kv4_ks(D, r)));
#pragma unroll
        for (int q = 0; q < D / 64; ++q) b[q] = scale[q];
      }
    }
  }
}

// ------------------------------------------------------------------ host side
size_t append_workspace(const Kv4& c, long long n_tokens, uint8_t* base, PlanWs* ws) {
  // a sequence needs at most one page per page_size new tokens, one for the remainder and one of its own
  const long long most = n_tokens / c.ps + 2ll * c.n_seqs;
  const int list = (int)(most < c.n_pages ? most : c.n_pages);
  const size_t row = kv4_align(4 * (size_t)c.n_seqs), l = 256 + 3 * row;
  if (ws) {
    *ws = {};
    ws->ok = (int32_t*)base;
    ws->len = (int32_t*)(base + 256);
    ws->off = (int32_t*)(base + 256 + row);
    ws->info = (int32_t*)(base + 256 + 2 * row);
    ws->list = (int32_t*)(base + l);
    ws->list_max = list;
  }
  return l + kv4_align(4 * (size_t)list);
}

int compact_cap(const Kv4& c, int keep_stride) {
  const long long cap = (long long)c.max_pages * c.ps;
  return (int)(cap < keep_stride ? cap : keep_stride);
}
size_t compact_workspace(const Kv4& c, int keep_stride, uint8_t* base, PlanWs* ws) {
  const int cap = compact_cap(c, keep_stride);
  const long long most = (long long)c.n_seqs * ((cap + c.ps - 1) / c.ps);
  const int list = (int)(most < c.n_pages ? most : c.n_pages);
  const size_t row = kv4_align(4 * (size_t)c.n_seqs);
  const size_t l = 256 + 5 * row + 256, s = l + kv4_align(4 * (size_t)list);
  if (ws) {
    *ws = {};
    ws->ok = (int32_t*)base;
    ws->off = (int32_t*)(base + 256);
    ws->info = (int32_t*)(base + 256 + row);
    ws->cnt = (int32_t*)(base + 256 + 2 * row);
    ws->len = (int32_t*)(base + 256 + 3 * row);
    ws->goff = (int32_t*)(base + 256 + 4 * row);
    ws->list = (int32_t*)(base + l);
    ws->list_max = list;
    ws->src = (int32_t*)(base + s);
    ws->cap = cap;
  }
  return s + kv4_align(4 * (size_t)c.n_seqs * cap);
}

bool overlap(const void* a, const void* b, size_t bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + bytes && y < x + bytes;
}
// `from` and `to` are the same arrays or apart, array by array
int check_maps(const Kv4& c, const im_kv4_map* from, const im_kv4_map* to, const char* fn, bool rows_apart) {
  int rc = kv4_check_map(from, fn);
  if (rc == IM_OK) rc = kv4_check_map(to, fn);
  if (rc != IM_OK) return rc;
  const size_t table = 4 * (size_t)c.n_seqs * c.max_pages, lens = 4 * (size_t)c.n_seqs, refs = 4 * (size_t)c.n_pages;
  const bool t = overlap(from->table, to->table, table), l = overlap(from->lens, to->lens, lens), r = overlap(from->refs, to->refs, refs);
  if (rows_apart && (t || l)) return kv4_fail(IM_ERR_ARG, fn, "table and lens of `to` must not overlap those of `from`");
  if ((t && from->table != to->table) || (l && from->lens != to->lens) || (r && from->refs != to->refs))
    return kv4_fail(IM_ERR_ARG, fn, "`to` must be `from` or not overlap it");
  return IM_OK;
}
// One CTA for pools it counts in a few rounds (no cluster barriers), else a cluster.
template <typename... KArgs, typename... Args>
cudaError_t launch_plan(void (*kernel)(KArgs...), const Kv4& c, cudaStream_t s, bool dependent, Args... args) {
  cudaLaunchConfig_t cfg = {};
  const int ctas = c.n_pages <= PLAN_ONE_CTA_PAGES ? 1 : PLAN_CTAS;
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(PLAN_THREADS);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = dependent ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, (KArgs)args...);
}
int launched(cudaError_t e) { return e == cudaSuccess ? IM_OK : im_fail_message(IM_ERR_CUDA, cudaGetErrorString(e)); }

}  // namespace

int kv4_fail(int code, const char* fn, const char* what) {
  char msg[240];
  snprintf(msg, sizeof(msg), "%s: %s", fn, what);
  return im_fail_message(code, msg);
}

extern "C" size_t im_kv4_page_bytes(int n_kv_heads, int head_dim, int page_size) {
  if (n_kv_heads < 1 || n_kv_heads > 256) return 0;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return 0;
  if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128) return 0;
  return (size_t)n_kv_heads * (page_size / 16) * kv4_group_bytes(head_dim);
}

int kv4_describe(const im_kv4* p, const char* fn, Kv4* out) {
  if (!p || !p->pool || !p->status) return kv4_fail(IM_ERR_ARG, fn, "null cache, pool or status");
  if ((uintptr_t)p->pool & 15) return kv4_fail(IM_ERR_ARG, fn, "the pool must be 16-byte aligned");
  if (!im_kv4_page_bytes(p->n_kv_heads, p->head_dim, p->page_size))
    return kv4_fail(IM_ERR_ARG, fn, "head_dim must be 64, 128 or 256, page_size 16, 32, 64 or 128, n_kv_heads 1 to 256");
  // 2^16 below 31 bits: the kernels round lengths up to their tiles (up to 16384 entries) in 32 bits
  if (p->n_pages < 1 || (long long)p->n_pages * p->page_size > 0x7fff0000ll || p->max_pages < 1 ||
      (long long)p->max_pages * p->page_size > 0x7fff0000ll || p->n_seqs < 1 || p->n_seqs > KV4_MAX_SEQS ||
      (double)p->max_pages * p->page_size * p->n_kv_heads * p->n_seqs > 68719476736.0)
    return kv4_fail(IM_ERR_ARG, fn, "n_pages, max_pages or n_seqs out of range");
  *out = {(uint8_t*)p->pool, p->k_exp, p->v_exp, p->status, p->n_pages, p->page_size, p->n_kv_heads, p->head_dim, p->n_seqs, p->max_pages};
  return IM_OK;
}

int kv4_check_map(const im_kv4_map* m, const char* fn) {
  if (!m || !m->refs || !m->table || !m->lens) return kv4_fail(IM_ERR_ARG, fn, "null map");
  if (((uintptr_t)m->refs | (uintptr_t)m->table | (uintptr_t)m->lens) & 3) return kv4_fail(IM_ERR_ARG, fn, "a map's arrays must be 4-byte aligned");
  return IM_OK;
}

extern "C" size_t im_kv4_workspace_bytes(const im_kv4* cache, int op, int n, int n_q_heads) {
  Kv4 c;
  if (kv4_describe(cache, "im_kv4_workspace_bytes", &c) != IM_OK) return 0;
  if (n < 0 || op < 0 || op > 2) return (size_t)(kv4_fail(IM_ERR_ARG, "im_kv4_workspace_bytes", "bad op or size"), 0);
  if (op == 0) return append_workspace(c, n, nullptr, nullptr);
  if (op == 2) return compact_workspace(c, n, nullptr, nullptr);
  if (n_q_heads < 1 || n_q_heads % c.Hkv) return (size_t)(kv4_fail(IM_ERR_ARG, "im_kv4_workspace_bytes", "bad n_q_heads"), 0);
  return kv4_attention_workspace(c, n, n_q_heads);
}

extern "C" int im_kv4_append(const im_kv4* cache, const im_kv4_map* from, const im_kv4_map* to, int dtype, const void* k,
                             long long k_stride, const void* v, long long v_stride, int n_tokens, const int32_t* cu_new,
                             void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const char* fn = "im_kv4_append";
  Kv4 c;
  int rc = kv4_describe(cache, fn, &c);
  if (rc == IM_OK) rc = check_maps(c, from, to, fn, false);
  if (rc != IM_OK) return rc;
  const long long dense = (long long)c.Hkv * c.d;
  if (!k_stride) k_stride = dense;
  if (!v_stride) v_stride = dense;
  if (dtype != IM_BF16 && dtype != IM_F16) return kv4_fail(IM_ERR_ARG, fn, "keys and values are bf16 or f16");
  if (n_tokens < 0 || (n_tokens > 0 && (!k || !v)) || (!cu_new && n_tokens != c.n_seqs))
    return kv4_fail(IM_ERR_ARG, fn, "null tensor or bad token count");
  if (k_stride < dense || v_stride < dense || (k_stride | v_stride) % 8 || (((uintptr_t)k | (uintptr_t)v) & 15))
    return kv4_fail(IM_ERR_ARG, fn, "token strides must be multiples of 8 elements, no shorter than a token; bases 16-byte aligned");
  PlanWs ws;
  if (!workspace || ((uintptr_t)workspace & 255) || append_workspace(c, n_tokens, (uint8_t*)workspace, &ws) > workspace_bytes)
    return kv4_fail(IM_ERR_CAPACITY, fn, "workspace missing, misaligned or too small");
  if ((long long)n_tokens * (c.d / 16) > 0x7fffff00ll) return kv4_fail(IM_ERR_ARG, fn, "too many tokens in one call");
  cudaStream_t s = (cudaStream_t)cuda_stream;
  cudaError_t e = launch_plan(k_kv4_plan<PLAN_APPEND>, c, s, false, c, *from, *to, cu_new, n_tokens, ws);
  if (e == cudaSuccess && n_tokens > 0) {
    const int x = (n_tokens * (c.d / 16) + STORE_THREADS - 1) / STORE_THREADS;
    const long long tasks = (long long)c.n_seqs * c.Hkv, copiers = tasks < 592 ? tasks : 592;  // (four blocks per SM)
    const dim3 grid(x, c.Hkv + (int)((copiers + x - 1) / x));
    if (dtype == IM_BF16)
      e = kv4_launch(k_kv4_store<bf16>, grid, STORE_THREADS, 0, s, true, c, to->table, to->lens, (const bf16*)k, k_stride, (const bf16*)v,
                     v_stride, n_tokens, cu_new, ws);
    else
      e = kv4_launch(k_kv4_store<__half>, grid, STORE_THREADS, 0, s, true, c, to->table, to->lens, (const __half*)k, k_stride,
                     (const __half*)v, v_stride, n_tokens, cu_new, ws);
  }
  return launched(e);
}

extern "C" int im_kv4_gather(const im_kv4* cache, const im_kv4_map* map, int n_rows, const int32_t* cu_rows, const int32_t* slots,
                             int dtype, void* k, void* v, void* cuda_stream) {
  const char* fn = "im_kv4_gather";
  Kv4 c;
  int rc = kv4_describe(cache, fn, &c);
  if (rc == IM_OK) rc = kv4_check_map(map, fn);
  if (rc != IM_OK) return rc;
  if (n_rows < 0 || (!cu_rows && n_rows != c.n_seqs)) return kv4_fail(IM_ERR_ARG, fn, "bad row count");
  if (dtype != IM_BF16 && dtype != IM_F16 && dtype != IM_F32) return kv4_fail(IM_ERR_ARG, fn, "unknown dtype");
  if ((!k && !v && n_rows) || (((uintptr_t)k | (uintptr_t)v) & 15)) return kv4_fail(IM_ERR_ARG, fn, "null or misaligned output");
  const long long blocks = ((long long)n_rows * c.Hkv * (c.d / 8) + GATHER_THREADS - 1) / GATHER_THREADS;
  if (blocks > 0xffffffffll / GATHER_THREADS) return kv4_fail(IM_ERR_ARG, fn, "too many rows in one call");
  if (!blocks) return IM_OK;
  const dim3 grid((unsigned)blocks);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  if (dtype == IM_BF16)
    return launched(kv4_launch(k_kv4_gather<bf16>, grid, GATHER_THREADS, 0, s, false, c, map->table, map->lens, n_rows, cu_rows, slots, (bf16*)k, (bf16*)v));
  if (dtype == IM_F16)
    return launched(kv4_launch(k_kv4_gather<__half>, grid, GATHER_THREADS, 0, s, false, c, map->table, map->lens, n_rows, cu_rows, slots, (__half*)k, (__half*)v));
  return launched(kv4_launch(k_kv4_gather<float>, grid, GATHER_THREADS, 0, s, false, c, map->table, map->lens, n_rows, cu_rows, slots, (float*)k, (float*)v));
}

extern "C" int im_kv4_fork(const im_kv4* cache, const im_kv4_map* from, const im_kv4_map* to, const int32_t* parent, void* cuda_stream) {
  const char* fn = "im_kv4_fork";
  Kv4 c;
  int rc = kv4_describe(cache, fn, &c);
  if (rc == IM_OK) rc = check_maps(c, from, to, fn, true);
  if (rc != IM_OK) return rc;
  if (!parent) return kv4_fail(IM_ERR_ARG, fn, "null parent");
  cudaStream_t s = (cudaStream_t)cuda_stream;
  const bool apart = from->refs != to->refs;
  cudaError_t e = cudaSuccess;
  if (apart) {
    const int blocks = (c.n_pages + 255) / 256;
    e = kv4_launch(k_kv4_copy_refs, dim3(blocks < 1184 ? blocks : 1184), 256, 0, s, false, (const int32_t*)from->refs, to->refs, c.n_pages);
  }
  const int segs = (c.max_pages + FORK_SEG - 1) / FORK_SEG;
  const long long blocks = ((long long)segs * c.n_seqs + FORK_THREADS / 32 - 1) / (FORK_THREADS / 32);
  if (blocks > 0x7fffffffll) return kv4_fail(IM_ERR_ARG, fn, "map too large");
  if (e == cudaSuccess) e = kv4_launch(k_kv4_fork, dim3((unsigned)blocks), FORK_THREADS, 0, s, apart, c, *from, *to, parent, segs);
  return launched(e);
}

extern "C" int im_kv4_compact(const im_kv4* cache, const im_kv4_map* from, const im_kv4_map* to, const uint8_t* keep, int keep_stride,
                              void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const char* fn = "im_kv4_compact";
  Kv4 c;
  int rc = kv4_describe(cache, fn, &c);
  if (rc == IM_OK) rc = check_maps(c, from, to, fn, false);
  if (rc != IM_OK) return rc;
  if (!keep || keep_stride < 1) return kv4_fail(IM_ERR_ARG, fn, "null keep or bad stride");
  PlanWs ws;
  if (!workspace || ((uintptr_t)workspace & 255) || compact_workspace(c, keep_stride, (uint8_t*)workspace, &ws) > workspace_bytes)
    return kv4_fail(IM_ERR_CAPACITY, fn, "workspace missing, misaligned or too small");
  // eight blocks per SM, and no more than there can be groups
  const long long groups = (long long)((ws.cap + 15) / 16) * c.n_seqs;
  const int sms = kv4_sm_count();
  if (sms < 1) return kv4_fail(IM_ERR_CUDA, fn, "no usable CUDA device");
  cudaStream_t s = (cudaStream_t)cuda_stream;
  cudaError_t e = kv4_launch(k_kv4_scan, dim3(c.n_seqs), SCAN_THREADS, 0, s, false, c, *from, keep, keep_stride, ws);
  if (e == cudaSuccess) e = launch_plan(k_kv4_plan<PLAN_COMPACT>, c, s, true, c, *from, *to, (const int32_t*)nullptr, 0, ws);
  if (e == cudaSuccess) {
    const dim3 grid((unsigned)(groups < 8 * sms ? groups : 8 * sms));
    if (c.d == 64) e = kv4_launch(k_kv4_move<64>, grid, MOVE_THREADS, 0, s, true, c, (const int32_t*)to->table, ws);
    else if (c.d == 128) e = kv4_launch(k_kv4_move<128>, grid, MOVE_THREADS, 0, s, true, c, (const int32_t*)to->table, ws);
    else e = kv4_launch(k_kv4_move<256>, grid, MOVE_THREADS, 0, s, true, c, (const int32_t*)to->table, ws);
  }
  return launched(e);
}
