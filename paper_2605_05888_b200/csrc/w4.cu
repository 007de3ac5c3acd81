// 4-bit weights with group scales: making them from bf16 or fp32 weights, giving them back, and their products with a few
// rows (moe_w4_pack, moe_w4_unpack, moe_w4_matvec of include/moehub.h).
#include "row_stream.cuh"

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

struct W4MatvecParams {
  const void* codes;
  const __nv_bfloat16* scales;
  const __nv_bfloat16* x;
  const int* expert;
  __nv_bfloat16* y;
  int experts, N, C, M;
};

// Rows of x are taken `batch` at a time: 8 * NT of one matrix, or 32 of several; rows with the same matrix share its
// reading by eights.
template <int G, int NT>
__global__ void __launch_bounds__(RsSizes<W4<G>, NT>::THREADS, 1)
w4_matvec_kernel(const __grid_constant__ W4MatvecParams p, int batch) {
  typedef RsSizes<W4<G>, NT> Z;
  constexpr int SLOTS = 8 * NT;
  extern __shared__ __align__(128) unsigned char dynamic[];
  __shared__ unsigned short used[32];
  __shared__ unsigned char count[32], token[32 * SLOTS];
  __shared__ int entries;
  float* slots = reinterpret_cast<float*>(dynamic + Z::RING);
  const uint32_t ring = smem_u32(dynamic) + threadIdx.x / 32 * (Z::STAGES * Z::STAGE);
  const int lane = threadIdx.x % 32;
  for (int m0 = 0; m0 < p.M; m0 += batch) {
    const int rows = min(batch, p.M - m0);
    if (threadIdx.x < 32) {  // an entry per matrix and SLOTS rows of it, in the order of their first rows
      int e = lane < rows ? p.expert != nullptr ? p.expert[m0 + lane] : 0 : -1;
      if (e < 0 || e >= p.experts) e = -1;
      const unsigned same = __match_any_sync(0xffffffffu, e);
      const int rank = __popc(same & ((1u << lane) - 1u));
      const bool first = e >= 0 && rank % SLOTS == 0;
      const unsigned firsts = __ballot_sync(0xffffffffu, first);
      const int mine = __popc(firsts & ((1u << lane) - 1u));
      const unsigned before = same & firsts & (0xffffffffu >> (31 - lane));  // the last of them begins this row's entry
      const int entry = __shfl_sync(0xffffffffu, mine, before != 0 ? 31 - __clz(before) : lane);
      if (first) {
        used[entry] = (unsigned short)e;
        count[entry] = (unsigned char)min(SLOTS, __popc(same) - rank);
      }
      if (e >= 0) token[entry * SLOTS + rank % SLOTS] = (unsigned char)lane;
      if (lane == 0) entries = __popc(firsts);
    }
    __syncthreads();
    const RsList list{used, count, token, entries};
    const RsOperand op{p.codes, p.codes, p.scales, p.scales, p.x + (size_t)m0 * p.C, p.N, p.C, p.experts};
    typedef RowStream<W4<G>, NT, kRsRows> Stream;
    Stream rs(op, list, ring);
    auto finish = [&](int u, int row, int n0, int n1, const float*) {
#pragma unroll
      for (int j = 0; j < Z::REGS; ++j) {
        const int t = rs.token(j), r = rs.row_of(j);
        const bool second = rs.run_of(j) == 1;
        if (t < count[u] && r < (second ? n1 : n0))
          p.y[(size_t)(m0 + token[u * SLOTS + t]) * p.N + row + (second ? n0 : 0) + r] = __float2bfloat16_rn(rs.acc[j]);
      }
    };
    rs.run(nullptr, slots, [](int, int) { return 0.0f; }, finish);
    __syncthreads();
    rs.join(slots, finish);
    __syncthreads();
  }
}

template <int G, int NT>
static cudaError_t launch_matvec(const W4MatvecParams& q, cudaStream_t st) {
  static SmemAttrOnce once;
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e == cudaSuccess) e = ensure_dynamic_smem(w4_matvec_kernel<G, NT>, RsSizes<W4<G>, NT>::BYTES, device, once);
  if (e != cudaSuccess) return e;
  const int sms = sm_count_now();
  if (sms <= 0) return cudaErrorUnknown;
  w4_matvec_kernel<G, NT><<<sms, RsSizes<W4<G>, NT>::THREADS, RsSizes<W4<G>, NT>::BYTES, st>>>(q, q.experts > 1 ? 32 : 8 * NT);
  return cudaGetLastError();
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
  if (experts > 65535 || C > (1 << 25)) return MOE_ERR_UNSUPPORTED;  // (16-bit matrix numbers, 32-bit offsets into a batch of x)
  if (((reinterpret_cast<uintptr_t>(d_x) | reinterpret_cast<uintptr_t>(d_y)) & 15) || (reinterpret_cast<uintptr_t>(d_expert) & 3))
    return MOE_ERR_ALIGN;
  const W4MatvecParams q{w->codes, (const __nv_bfloat16*)w->scales, (const __nv_bfloat16*)d_x, d_expert, (__nv_bfloat16*)d_y, experts, N, C, M};
  cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e;
  if (M <= 8 || experts > 1) e = group == 32 ? launch_matvec<32, 1>(q, st) : group == 64 ? launch_matvec<64, 1>(q, st) : launch_matvec<128, 1>(q, st);
  else e = group == 32 ? launch_matvec<32, 2>(q, st) : group == 64 ? launch_matvec<64, 2>(q, st) : launch_matvec<128, 2>(q, st);
  return e == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

}  // extern "C"
