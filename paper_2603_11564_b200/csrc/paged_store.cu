// Rows into pages and back: appending tokens with their rotation, an eviction's retained rows, reading rows as values.
// All three move bytes (a row of 128 channels is 256 bytes in bf16, 512 in fp32, 72 in 4 bits); what they compute is hidden behind
// the loads.
#include "paged.cuh"

namespace dapq {
namespace {

constexpr int kStoreThreads = 256, kLanes = 16;        // 16 threads a row: channels 4 l .. 4 l + 3 and 64 + 4 l .. 64 + 4 l + 3
constexpr int kHalf = kHeadDim / 2;

struct Eight { float lo[4], hi[4]; };

__device__ __forceinline__ float4 load4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
__device__ __forceinline__ uint2 load4(const __nv_bfloat16* p) { return __ldg(reinterpret_cast<const uint2*>(p)); }
__device__ __forceinline__ void widen(float4 x, float* y) { y[0] = x.x; y[1] = x.y; y[2] = x.z; y[3] = x.w; }
__device__ __forceinline__ void widen(uint2 x, float* y) {
  y[0] = __uint_as_float(x.x << 16);
  y[1] = __uint_as_float(x.x & 0xffff0000u);
  y[2] = __uint_as_float(x.y << 16);
  y[3] = __uint_as_float(x.y & 0xffff0000u);
}
template <typename T> struct Raw { decltype(load4((const T*)nullptr)) lo, hi; };
template <typename T> __device__ __forceinline__ Raw<T> load_row(const T* row, int lane) { return {load4(row + 4 * lane), load4(row + kHalf + 4 * lane)}; }
template <typename T> __device__ __forceinline__ Eight widen_row(const Raw<T>& r) {
  Eight x;
  widen(r.lo, x.lo);
  widen(r.hi, x.hi);
  return x;
}
__device__ __forceinline__ void store4(float* p, const float* x) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float* x) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// Four channels of each of a row's halves in 4 bits; four lanes hold a group of 16.  Every rounding is that of the formula: the
// quotients x / (scale kappa) are correctly rounded (reciprocal, product and one correction by the exact remainder, after
// Markstein 1990), so ties go where they would in exact arithmetic whenever scale kappa is exact.  x is clamped to where the largest code
// already holds, which keeps the remainder finite.
__device__ __forceinline__ void store_fp4(char* codes, unsigned char* scales, float kappa, int64_t off, int lane, const float* x, int group_base, bool ok) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);      // (NaN above infinity above all numbers)
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const bool fine = top < 0x7f800000u;
  const __nv_fp8_storage_t s = __nv_cvt_float_to_fp8(fminf(__fdiv_rn(__uint_as_float(fine ? top : 0u), __fmul_rn(6.f, kappa)), 448.f), __NV_SATFINITE, __NV_E4M3);
  const float step = __fmul_rn(scale_to_float(s), kappa), r = __frcp_rn(step), most = 7.f * step;
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float v = fminf(fmaxf(x[i], -most), most), q = __fmul_rn(v, r);
    y[i] = step > 0.f && fine ? __fmaf_rn(__fmaf_rn(-q, step, v), r, q) : 0.f;
  }
  const uint32_t a = __nv_cvt_float2_to_fp4x2(make_float2(y[0], y[1]), __NV_E2M1, cudaRoundNearest);
  const uint32_t b = __nv_cvt_float2_to_fp4x2(make_float2(y[2], y[3]), __NV_E2M1, cudaRoundNearest);
  if (ok) {
    *reinterpret_cast<uint16_t*>(codes + off / 2 + group_base / 2 + 2 * lane) = (uint16_t)(a | (b << 8));
    if ((lane & 3) == 0) scales[off / 16 + group_base / 16 + lane / 4] = fine ? s : 0x7f;
  }
}

// One row of K (or V) to its place; all lanes of a warp come here together.
template <typename T, bool kFp4>
__device__ __forceinline__ void store_row(char* base, unsigned char* scales, float kappa, int64_t off, int lane, const Eight& x, bool ok) {
  if (kFp4) {
    store_fp4(base, scales, kappa, off, lane, x.lo, 0, ok);
    store_fp4(base, scales, kappa, off, lane, x.hi, kHalf, ok);
  } else if (ok) {
    store4(reinterpret_cast<T*>(base) + off + 4 * lane, x.lo);
    store4(reinterpret_cast<T*>(base) + off + kHalf + 4 * lane, x.hi);
  }
}

// The rotation in fp32, every product and sum rounded by itself: what a user's own elementwise rotation gives, bit for bit.
__device__ __forceinline__ float turn_lo(float lo, float hi, float2 cs) { return __fsub_rn(__fmul_rn(lo, cs.x), __fmul_rn(hi, cs.y)); }
__device__ __forceinline__ float turn_hi(float lo, float hi, float2 cs) { return __fadd_rn(__fmul_rn(hi, cs.x), __fmul_rn(lo, cs.y)); }
__device__ __forceinline__ void rotate(Eight& x, const float2* cs, int lane, int interleaved) {
  if (interleaved) {
    float* half[2] = {x.lo, x.hi};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const float2 a = cs[kHalf / 2 * h + 2 * lane + p];
        const float lo = half[h][2 * p], hi = half[h][2 * p + 1];
        half[h][2 * p] = turn_lo(lo, hi, a);
        half[h][2 * p + 1] = turn_hi(lo, hi, a);
      }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 a = cs[4 * lane + i];
      const float lo = x.lo[i], hi = x.hi[i];
      x.lo[i] = turn_lo(lo, hi, a);
      x.hi[i] = turn_hi(lo, hi, a);
    }
  }
}

// A block takes kTok consecutive tokens: it evaluates their angles once for all heads, then its 16 groups of 16 threads take the
// tokens' rows (K heads, V heads, query heads) in turn, kUnroll rows a group in flight.
constexpr int kUnroll = 4;
template <typename T, bool kFp4, int kTok>
__global__ void __launch_bounds__(kStoreThreads)
paged_append_kernel(const __grid_constant__ PagedDev pg, const __grid_constant__ NewRows t, const __grid_constant__ NewTokensDev nt,
                    const double* __restrict__ inv_freq, int n_kv_heads, int n_q_heads, int interleaved, int* __restrict__ status) {
  __shared__ float2 angle[kTok][kHalf];
  __shared__ int seq[kTok];
  __shared__ int64_t place[kTok];
  const int tok0 = blockIdx.x * kTok, n = min(kTok, t.cu[t.batch] - tok0);
  if (threadIdx.x < n) seq[threadIdx.x] = find_segment(t.cu, t.batch, tok0 + threadIdx.x);
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x < n) {
    const int b = seq[threadIdx.x], held = pg.len[b];
    int64_t off = -1;
    if (held >= 0) {
      off = paged_row(pg, b, (int64_t)held + (tok0 + threadIdx.x - t.cu[b]), 0);
      if (off < 0) atomicOr(status, kStatusBadPage);
    }
    place[threadIdx.x] = off;
  }
  if (nt.positions != nullptr)
    for (int a = threadIdx.x; a < n * kHalf; a += kStoreThreads) {
      double sn, cs;
      sincos((double)nt.positions[tok0 + a / kHalf] * inv_freq[a % kHalf], &sn, &cs);
      angle[a / kHalf][a % kHalf] = make_float2((float)cs, (float)sn);
    }
  __syncthreads();
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes, groups = kStoreThreads / kLanes;
  const int per_token = 2 * n_kv_heads + (nt.q != nullptr ? n_q_heads : 0), rows = n * per_token;
  for (int r0 = 0; r0 < rows; r0 += groups * kUnroll) {                 // (the same for the whole block)
    Raw<T> raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int r = min(r0 + u * groups + group, rows - 1), tk = r / per_token, h = r - tk * per_token;
      const int64_t at = tok0 + tk;
      const T* row = h < n_kv_heads       ? (const T*)nt.k + at * nt.k_stride + h * kHeadDim
                     : h < 2 * n_kv_heads ? (const T*)nt.v + at * nt.v_stride + (h - n_kv_heads) * kHeadDim
                                          : (const T*)nt.q + at * nt.q_stride + (h - 2 * n_kv_heads) * kHeadDim;
      raw[u] = load_row(row, lane);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int r = r0 + u * groups + group, rc = min(r, rows - 1), tk = rc / per_token, h = rc - tk * per_token;
      Eight x = widen_row<T>(raw[u]);
      const bool is_k = h < n_kv_heads, is_q = h >= 2 * n_kv_heads;
      if ((is_k || is_q) && nt.positions != nullptr) rotate(x, angle[tk], lane, interleaved);
      const bool ok = r < rows && !is_q && place[tk] >= 0;
      const int64_t off = place[tk] + (is_k ? h : h - n_kv_heads) * pg.head_stride;
      store_row<T, kFp4>(is_k ? pg.k : pg.v, is_k ? pg.k_scales : pg.v_scales, is_k ? pg.k_scale : pg.v_scale, off, lane, x, ok);
      if (is_q && r < rows)
        store_row<T, false>((char*)nt.q_rot, nullptr, 0.f, ((int64_t)(tok0 + tk) * n_q_heads + h - 2 * n_kv_heads) * kHeadDim, lane, x, true);
    }
  }
}

// Retained rows: a thread moves its channels of kKeep rows, of K and of V.
constexpr int kKeep = 2;
template <typename T, bool kFp4>
__global__ void __launch_bounds__(kStoreThreads)
paged_compact_kernel(const __grid_constant__ PagedDev pg, const __grid_constant__ CacheDev cv, const int32_t* __restrict__ idx,
                     const __grid_constant__ SeqTable t, int* __restrict__ status) {
  const int kt = t.cu_keep[t.batch], lane = threadIdx.x % kLanes, kvh = blockIdx.y;
  const int r0 = (int)(((int64_t)blockIdx.x * kStoreThreads + threadIdx.x) / kLanes) * kKeep;
  int seg[kKeep];
#pragma unroll
  for (int i = 0; i < kKeep; ++i) seg[i] = find_segment(t.cu_keep, t.batch, min(r0 + i, kt - 1));
  pdl_wait();
  pdl_trigger();
  Raw<T> k[kKeep], v[kKeep];
  int64_t off[kKeep];
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    const int r = min(r0 + i, kt - 1), b = seg[i], held = pg.len[b];
    const int32_t j = idx[(int64_t)kvh * kt + r];
    const bool in = j >= 0 && j < t.prompt_len[b];              // never read outside the sequence's prompt rows
    const bool mine = r0 + i < kt && held >= 0;
    off[i] = mine ? paged_row(pg, b, (int64_t)held + (r - t.cu_keep[b]), kvh) : -1;
    if (mine && (!in || off[i] < 0) && lane == 0) atomicOr(status, in ? kStatusBadPage : kStatusBadIndex);
    if (!in) off[i] = -1;
    const int64_t row = t.cu_rows[b] + (in ? j : 0);
    k[i] = load_row((const T*)cv.k + (int64_t)kvh * cv.k_head_stride + row * cv.k_row_stride, lane);
    v[i] = load_row((const T*)cv.v + (int64_t)kvh * cv.v_head_stride + row * cv.v_row_stride, lane);
  }
#pragma unroll
  for (int i = 0; i < kKeep; ++i) {
    store_row<T, kFp4>(pg.k, pg.k_scales, pg.k_scale, off[i], lane, widen_row<T>(k[i]), off[i] >= 0);
    store_row<T, kFp4>(pg.v, pg.v_scales, pg.v_scale, off[i], lane, widen_row<T>(v[i]), off[i] >= 0);
  }
}

// Rows as values: a thread holds a group of 16 channels, of K and of V.
constexpr int kGroup = 16, kGroups = kHeadDim / kGroup;
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float* x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    __nv_bfloat162 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __floats2bfloat162_rn(x[8 * h + 2 * i], x[8 * h + 2 * i + 1]);
    reinterpret_cast<uint4*>(p)[h] = *reinterpret_cast<const uint4*>(w);
  }
}
__device__ __forceinline__ void store16(float* p, const float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) store4(p + 4 * i, x + 4 * i);
}
template <typename T, bool kFp4>
__global__ void __launch_bounds__(kStoreThreads)
paged_read_kernel(const __grid_constant__ PagedDev pg, const __grid_constant__ ReadRows t, T* __restrict__ k_out, T* __restrict__ v_out,
                  int64_t out_head_stride, int* __restrict__ status) {
  const int total = t.rows.cu[t.rows.batch], kvh = blockIdx.y;
  const int64_t gid = (int64_t)blockIdx.x * kStoreThreads + threadIdx.x;
  const int r = (int)(gid / kGroups), c = (int)(gid % kGroups) * kGroup;
  pdl_wait();
  pdl_trigger();
  if (r >= total) return;
  const int b = find_segment(t.rows.cu, t.rows.batch, r), i = r - t.rows.cu[b];
  const int64_t off = paged_row(pg, b, (int64_t)t.first[b] + i, kvh);
  const int64_t to = kvh * out_head_stride + ((int64_t)t.row_at[b] + i) * kHeadDim + c;
  constexpr int kWords = kGroup * sizeof(T) / 16;
  uint4* out[2] = {reinterpret_cast<uint4*>(k_out + to), reinterpret_cast<uint4*>(v_out + to)};
  if (off < 0) {
    if (c == 0) atomicOr(status, kStatusBadPage);
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int w = 0; w < kWords; ++w) out[p][w] = make_uint4(0, 0, 0, 0);
    return;
  }
  if (kFp4) {
    const uint2 code[2] = {__ldg(reinterpret_cast<const uint2*>(pg.k + (off + c) / 2)), __ldg(reinterpret_cast<const uint2*>(pg.v + (off + c) / 2))};
    const unsigned char scale[2] = {__ldg(pg.k_scales + (off + c) / 16), __ldg(pg.v_scales + (off + c) / 16)};
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const float s = scale_to_float(scale[p]), kappa = p == 0 ? pg.k_scale : pg.v_scale;
      float x[kGroup];
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const float2 y = __half22float2(fp4x2_to_half2(((w < 4 ? code[p].x : code[p].y) >> (8 * (w & 3))) & 255u));
        x[2 * w] = __fmul_rn(__fmul_rn(y.x, s), kappa);
        x[2 * w + 1] = __fmul_rn(__fmul_rn(y.y, s), kappa);
      }
      store16(p == 0 ? k_out + to : v_out + to, x);
    }
  } else {
    const uint4* in[2] = {reinterpret_cast<const uint4*>((const T*)pg.k + off + c), reinterpret_cast<const uint4*>((const T*)pg.v + off + c)};
    uint4 x[2][kWords];
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int w = 0; w < kWords; ++w) x[p][w] = __ldg(in[p] + w);
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int w = 0; w < kWords; ++w) out[p][w] = x[p][w];
  }
}

// Calls fn with the kernel's element type and format as types.
template <class F>
void by_type(int dtype, int fp4, F&& fn) {
  if (dtype == DAPQ_BF16) fp4 ? fn((__nv_bfloat16*)nullptr, std::true_type()) : fn((__nv_bfloat16*)nullptr, std::false_type());
  else fp4 ? fn((float*)nullptr, std::true_type()) : fn((float*)nullptr, std::false_type());
}

}  // namespace

cudaError_t launch_paged_append(int dtype, const PagedDev& pg, const NewRows& t, const NewTokensDev& nt, const double* inv_freq_dev, const Dims& dm,
                                int* status, cudaStream_t s, LaunchLog* log) {
  const int n = t.cu[t.batch];
  log->begin(kKindPagedAppend, s);
  by_type(dtype, pg.fp4, [&](auto* type, auto fp4) {
    using T = std::remove_pointer_t<decltype(type)>;
    auto go = [&](auto kernel, int tok) {
      launch_pdl(kernel, dim3((n + tok - 1) / tok), dim3(kStoreThreads), 0, s, 1, pg, t, nt, inv_freq_dev, dm.n_kv_heads, dm.n_q_heads, dm.rope_interleaved, status);
    };
    if (n > 1024) go(paged_append_kernel<T, decltype(fp4)::value, 4>, 4);
    else go(paged_append_kernel<T, decltype(fp4)::value, 1>, 1);
  });
  log->end(s);
  return cudaGetLastError();
}

cudaError_t launch_paged_compact(int dtype, const PagedDev& pg, const CacheDev& cv, const int32_t* idx, const SeqTable& t, int n_kv_heads, int* status,
                                 cudaStream_t s, LaunchLog* log) {
  const int rows_per_block = kStoreThreads / kLanes * kKeep;
  const dim3 grid((t.cu_keep[t.batch] + rows_per_block - 1) / rows_per_block, n_kv_heads);
  log->begin(kKindCompact, s);
  by_type(dtype, pg.fp4, [&](auto* type, auto fp4) {
    using T = std::remove_pointer_t<decltype(type)>;
    launch_pdl(paged_compact_kernel<T, decltype(fp4)::value>, grid, dim3(kStoreThreads), 0, s, 1, pg, cv, idx, t, status);
  });
  log->end(s);
  return cudaGetLastError();
}

cudaError_t launch_paged_read(int dtype, const PagedDev& pg, const ReadRows& t, int n_kv_heads, void* k_out, void* v_out, int64_t out_head_stride,
                              int* status, cudaStream_t s, LaunchLog* log) {
  const dim3 grid((unsigned)(((int64_t)t.rows.cu[t.rows.batch] * kGroups + kStoreThreads - 1) / kStoreThreads), n_kv_heads);
  log->begin(kKindPagedRead, s);
  by_type(dtype, pg.fp4, [&](auto* type, auto fp4) {
    using T = std::remove_pointer_t<decltype(type)>;
    launch_pdl(paged_read_kernel<T, decltype(fp4)::value>, grid, dim3(kStoreThreads), 0, s, 1, pg, t, (T*)k_out, (T*)v_out, out_head_stride, status);
  });
  log->end(s);
  return cudaGetLastError();
}

}  // namespace dapq
