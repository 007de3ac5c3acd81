// 4-bit weights with group scales: making them from bf16 or fp32 weights, giving them back, and their products with a few
// rows (moe_w4_pack, moe_w4_unpack, moe_w4_matvec of include/moehub.h).
#include "w4_common.cuh"

namespace moehub {

constexpr int kPackThreads = 256;

template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <> __device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
  Vec16<float>::unpack(__ldcs(reinterpret_cast<const uint4*>(p)), v);
  Vec16<float>::unpack(__ldcs(reinterpret_cast<const uint4*>(p) + 1), v + 4);
}
template <> __device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float (&v)[8]) {
  Vec16<__nv_bfloat16>::unpack(__ldcs(reinterpret_cast<const uint4*>(p)), v);
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]);
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&v)[8]) {
  __stcs(reinterpret_cast<uint4*>(p), Vec16<float>::pack(v));
  __stcs(reinterpret_cast<uint4*>(p) + 1, Vec16<float>::pack(v + 4));
}
template <> __device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, const float (&v)[8]) {
  __stcs(reinterpret_cast<uint4*>(p), Vec16<__nv_bfloat16>::pack(v));
}

// The code of w (the nearest integer to w / s, ties to even, within -8..7, plus 8).  The quotient in fp32 can land on the
// border between two integers without w doing so, so the decision is left to the remainder w - k s: k s has at most 12 bits and
// lies within s of w, so the fused multiply-add gives it exactly.
__device__ __forceinline__ uint32_t w4_code(float w, float s) {
  if (!(s > 0.0f) || !(s < INFINITY)) return 8u;
  const float k = rintf(fminf(fmaxf(w / s, -9.0f), 9.0f));
  const float r = __fmaf_rn(-k, s, w), half = 0.5f * s;
  int q = (int)k;
  if (r > half || (r == half && (q & 1))) q += 1;
  if (r < -half || (r == -half && (q & 1))) q -= 1;
  return (uint32_t)(min(max(q, -8), 7) + 8);
}

// A thread takes the eight columns of a word, neighbouring threads neighbouring words of a row; the G / 8 threads of a group
// find its largest magnitude together.
template <typename T, int G>
__global__ void __launch_bounds__(kPackThreads)
w4_pack_kernel(const T* __restrict__ w, size_t words, int N, int C, uint32_t* __restrict__ codes, __nv_bfloat16* __restrict__ scales) {
  constexpr int LANES = G / 8;
  const int per_row = C / 8;
  for (size_t i0 = (size_t)blockIdx.x * kPackThreads; i0 < words; i0 += (size_t)gridDim.x * kPackThreads) {
    const size_t i = i0 + threadIdx.x;
    const bool live = i < words;  // (whole groups: words is a multiple of LANES)
    float v[8];
    if (live) load8(w + i * 8, v);
    float largest = 0.0f;
    bool fine = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (!live) v[j] = 0.0f;
      largest = fmaxf(largest, fabsf(v[j]));
      fine = fine && fabsf(v[j]) < INFINITY;
    }
    if (!fine) largest = INFINITY;  // a NaN or an infinity: the group's scale is NaN
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, off));
    const __nv_bfloat16 scale = __float2bfloat16_rn(largest < INFINITY ? __fdiv_rn(largest, 7.0f) : __int_as_float(0x7fc00000));
    if (!live) continue;
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) word |= w4_code(v[j], __bfloat162float(scale)) << w4_shift(j);
    codes[i] = word;
    if (threadIdx.x % LANES == 0) {
      const size_t row = i / per_row;  // of all the experts' rows
      const int g = (int)(i % per_row) / LANES;
      scales[(row / N * (C / G) + g) * N + row % N] = scale;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kPackThreads)
w4_unpack_kernel(const uint32_t* __restrict__ codes, const __nv_bfloat16* __restrict__ scales, size_t words, int N, int C, int G, T* __restrict__ w) {
  const int per_row = C / 8, per_group = G / 8;
  for (size_t i = (size_t)blockIdx.x * kPackThreads + threadIdx.x; i < words; i += (size_t)gridDim.x * kPackThreads) {
    const size_t row = i / per_row;
    const int g = (int)(i % per_row) / per_group;
    const float scale = __bfloat162float(scales[(row / N * (C / G) + g) * N + row % N]);
    const uint32_t word = __ldcs(codes + i);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = scale * w4_value(word, j);
    store8(w + i * 8, v);
  }
}

static int sm_count_now() {
  int device = 0, sms = 0;
  if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return 0;
  return sms;
}

static int pack_grid(size_t words) {
  const size_t want = (words + kPackThreads - 1) / kPackThreads;
  const size_t most = (size_t)sm_count_now() * 8;
  return (int)(want < most ? want : most);
}

template <typename T>
static cudaError_t launch_pack(const void* w, size_t words, int N, int C, int group, const moe_w4_t& out, cudaStream_t st) {
  const int grid = pack_grid(words);
  if (grid <= 0) return cudaErrorUnknown;
  auto kern = group == 32 ? w4_pack_kernel<T, 32> : group == 64 ? w4_pack_kernel<T, 64> : w4_pack_kernel<T, 128>;
  kern<<<grid, kPackThreads, 0, st>>>((const T*)w, words, N, C, (uint32_t*)out.codes, (__nv_bfloat16*)out.scales);
  return cudaGetLastError();
}

template <typename T>
static cudaError_t launch_unpack(const moe_w4_t& w, size_t words, int N, int C, int group, void* out, cudaStream_t st) {
  const int grid = pack_grid(words);
  if (grid <= 0) return cudaErrorUnknown;
  w4_unpack_kernel<T><<<grid, kPackThreads, 0, st>>>((const uint32_t*)w.codes, (const __nv_bfloat16*)w.scales, words, N, C, group, (T*)out);
  return cudaGetLastError();
}

// ---- products with a few rows ------------------------------------------------------------------------------------------------

constexpr int kMatvecThreads = 256;

// A warp per result: lanes over the row's words.
__global__ void __launch_bounds__(kMatvecThreads)
w4_matvec_kernel(const uint32_t* __restrict__ codes, const __nv_bfloat16* __restrict__ scales, int experts, int N, int C, int G,
                 const __nv_bfloat16* __restrict__ x, const int* __restrict__ expert, int M, __nv_bfloat16* __restrict__ y) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, per_row = C / 8;
  for (int m = blockIdx.y; m < M; m += gridDim.y) {
    const int e = expert == nullptr ? 0 : expert[m];
    if (e < 0 || e >= experts) continue;
    for (int n = blockIdx.x * (kMatvecThreads / 32) + warp; n < N; n += gridDim.x * (kMatvecThreads / 32)) {
      float acc = 0.0f;
      for (int i = lane; i < per_row; i += 32) {
        const uint32_t word = __ldg(codes + ((size_t)e * N + n) * per_row + i);
        const float scale = __bfloat162float(scales[((size_t)e * (C / G) + i * 8 / G) * N + n]);
        float v[8], part = 0.0f;
        Vec16<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(x + (size_t)m * C + i * 8), v);
#pragma unroll
        for (int j = 0; j < 8; ++j) part = __fmaf_rn(w4_value(word, j), v[j], part);
        acc = __fmaf_rn(scale, part, acc);
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, off);
      if (lane == 0) y[(size_t)m * N + n] = __float2bfloat16_rn(acc);
    }
  }
}

}  // namespace moehub

using namespace moehub;

extern "C" {

int moe_w4_pack(int32_t dtype, int32_t experts, int32_t N, int32_t C, int32_t group, const void* d_w, const moe_w4_t* out, void* stream) {
  if (dtype != MOE_DTYPE_FP32 && dtype != MOE_DTYPE_BF16) return MOE_ERR_ARG;
  int rc = w4_check(out, experts, N, C, group);
  if (rc != MOE_OK) return rc;
  if (!d_w) return MOE_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(d_w) & 15) return MOE_ERR_ALIGN;
  const size_t words = (size_t)experts * N * (C / 8);
  cudaError_t e = dtype == MOE_DTYPE_FP32 ? launch_pack<float>(d_w, words, N, C, group, *out, (cudaStream_t)stream)
                                          : launch_pack<__nv_bfloat16>(d_w, words, N, C, group, *out, (cudaStream_t)stream);
  return e == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

int moe_w4_unpack(int32_t dtype, int32_t experts, int32_t N, int32_t C, int32_t group, const moe_w4_t* w, void* d_out, void* stream) {
  if (dtype != MOE_DTYPE_FP32 && dtype != MOE_DTYPE_BF16) return MOE_ERR_ARG;
  int rc = w4_check(w, experts, N, C, group);
  if (rc != MOE_OK) return rc;
  if (!d_out) return MOE_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(d_out) & 15) return MOE_ERR_ALIGN;
  const size_t words = (size_t)experts * N * (C / 8);
  cudaError_t e = dtype == MOE_DTYPE_FP32 ? launch_unpack<float>(*w, words, N, C, group, d_out, (cudaStream_t)stream)
                                          : launch_unpack<__nv_bfloat16>(*w, words, N, C, group, d_out, (cudaStream_t)stream);
  return e == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

int moe_w4_matvec(int32_t experts, int32_t N, int32_t C, int32_t group, const moe_w4_t* w, int32_t M, const void* d_x,
                  const int32_t* d_expert, void* d_y, void* stream) {
  int rc = w4_check(w, experts, N, C, group);
  if (rc != MOE_OK) return rc;
  if (M < 0) return MOE_ERR_ARG;
  if (M == 0) return MOE_OK;
  if (!d_x || !d_y || (experts > 1 && !d_expert)) return MOE_ERR_ARG;
  if (((reinterpret_cast<uintptr_t>(d_x) | reinterpret_cast<uintptr_t>(d_y)) & 15) || (reinterpret_cast<uintptr_t>(d_expert) & 3))
    return MOE_ERR_ALIGN;
  const dim3 grid(min((N + 7) / 8, 148 * 8), min(M, 65535));
  w4_matvec_kernel<<<grid, kMatvecThreads, 0, (cudaStream_t)stream>>>((const uint32_t*)w->codes, (const __nv_bfloat16*)w->scales, experts, N, C, group,
                                                                      (const __nv_bfloat16*)d_x, d_expert, M, (__nv_bfloat16*)d_y);
  return cudaGetLastError() == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

}  // extern "C"
