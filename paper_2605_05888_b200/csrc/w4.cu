// 4-bit weights with group scales: making them from bf16 or fp32 weights, giving them back, and their products with a few
// rows (moe_w4_pack, moe_w4_unpack, moe_w4_matvec of include/moehub.h).
#include "row_stream.cuh"

namespace moehub {

// ---- packing and unpacking: bound by HBM; a warp (of short rows: a part of one) walks along a row, so that a row's place is
// worked out once, with kPackUnroll words of eight columns per lane in flight ------------------------------------------------------
constexpr int kPackThreads = 256;
constexpr int kPackUnroll = 4;

template <typename T> struct Eight;  // eight columns
template <> struct Eight<float> {
  uint4 v[2];
  __device__ __forceinline__ void load(const float* p) {
    v[0] = __ldcs(reinterpret_cast<const uint4*>(p));
    v[1] = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
  }
  __device__ __forceinline__ void floats(float (&f)[8]) const {
    Vec16<float>::unpack(v[0], f);
    Vec16<float>::unpack(v[1], f + 4);
  }
};
template <> struct Eight<__nv_bfloat16> {
  uint4 v[1];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v[0] = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void floats(float (&f)[8]) const { Vec16<__nv_bfloat16>::unpack(v[0], f); }
};

// The code of w (the nearest integer to w / s, ties to even, within -8..7, plus 8); inverse: 1 / s.  A product with the inverse and one
// correction give the quotient rounded to fp32, which is exact where w / s lies on the border between two codes.  Where w is a
// bf16 number it is nowhere else on a border ((2 k + 1) s / 2 has 12 bits, w 8: they are equal, or 2^-13 apart); where w is an fp32 number
// the decision is left to the remainder w - k s, which is exact: k s has 12 bits and lies within s of w.
template <bool BF16>
__device__ __forceinline__ uint32_t w4_code(float w, float s, float inverse) {
  const float near = w * inverse;
  const float quotient = __fmaf_rn(__fmaf_rn(-near, s, w), inverse, near);
  constexpr float kIntegers = 12582912.0f;  // 1.5 * 2^23: a sum with it is an integer, in the last bits
  float sum = quotient + (kIntegers + 8.0f);
  if (!BF16) {
    const float k = sum - (kIntegers + 8.0f), r = __fmaf_rn(-k, s, w), half = 0.5f * s;
    const bool odd = __float_as_uint(sum) & 1u;
    if (fabsf(r) > half || (fabsf(r) == half && odd)) sum += r > 0.0f ? 1.0f : -1.0f;
  }
  return min(__float_as_uint(sum) - 0x4b400000u, 15u);  // (the largest quotient is 7 and what the scale was rounded by)
}
// The same without assuming that s has an inverse.
__device__ __noinline__ uint32_t w4_code_tiny(float w, float s) {
  const double q = rint((double)w / (double)s);
  return (uint32_t)(int)(fmin(fmax(q, -8.0), 7.0) + 8.0);
}

struct PackRows {
  long long rows;  // of all the matrices
  int N, C, lanes; // lanes: per row, a power of two
};

template <typename T, int G>
__global__ void __launch_bounds__(kPackThreads)
w4_pack_kernel(const T* __restrict__ w, const PackRows p, uint32_t* __restrict__ codes, __nv_bfloat16* __restrict__ scales) {
  constexpr int LANES = G / 8;  // of a group
  const int per_row = p.C / 8, lane = threadIdx.x % p.lanes;
  const long long step = (long long)gridDim.x * kPackThreads / p.lanes;
  for (long long r0 = ((long long)blockIdx.x * kPackThreads + threadIdx.x) / p.lanes;; r0 += step) {
    const bool live = r0 < p.rows;
    if (!__any_sync(0xffffffffu, live)) break;
    const long long row = live ? r0 : 0;
    const long long e = row / p.N;
    const int n = (int)(row - e * p.N);
    const T* from = w + row * p.C;
    for (int i0 = lane; i0 - lane < per_row; i0 += p.lanes * kPackUnroll) {
      Eight<T> raw[kPackUnroll];
#pragma unroll
      for (int j = 0; j < kPackUnroll; ++j)
        if (live && i0 + j * p.lanes < per_row) raw[j].load(from + (size_t)(i0 + j * p.lanes) * 8);
#pragma unroll
      for (int j = 0; j < kPackUnroll; ++j) {
        const int i = i0 + j * p.lanes;
        const bool mine = live && i < per_row;  // (whole groups: per_row is a multiple of LANES)
        float v[8], largest = 0.0f;
        if (mine) raw[j].floats(v);
        bool fine = true;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          if (!mine) v[c] = 0.0f;
          largest = fmaxf(largest, fabsf(v[c]));
          fine = fine && !isnan(v[c]);
        }
        if (!fine) largest = INFINITY;  // a NaN or an infinity: the group's scale is NaN
#pragma unroll
        for (int off = LANES / 2; off > 0; off >>= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, off));
        const __nv_bfloat16 scale = __float2bfloat16_rn(largest < INFINITY ? __fdiv_rn(largest, 7.0f) : __int_as_float(0x7fc00000));
        if (!mine) continue;
        const float s = __bfloat162float(scale);
        uint32_t word = 0x88888888u;  // scale 0 or NaN
        if (s >= 1e-30f) {
          const float inverse = __frcp_rn(s);
          word = 0;
#pragma unroll
          for (int c = 0; c < 8; ++c) word |= w4_code<sizeof(T) == 2>(v[c], s, inverse) << w4_shift(c);
        } else if (s > 0.0f) {
          word = 0;
#pragma unroll 1
          for (int c = 0; c < 8; ++c) word |= w4_code_tiny(v[c], s) << w4_shift(c);
        }
        __stcs(codes + row * per_row + i, word);
        if (i % LANES == 0) scales[(e * (p.C / G) + i / LANES) * p.N + n] = scale;
      }
    }
  }
}

// Eight codes times their scale, rounded once.
__device__ __forceinline__ void w4_unpack8(uint32_t word, __nv_bfloat16 scale, __nv_bfloat16* to) {
  const __nv_bfloat162 s = __halves2bfloat162(scale, scale), bias = __halves2bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308));  // 136
  uint32_t d[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // columns 2 i and 2 i + 1: 128 + code, less 136
    const uint32_t v = ((word >> (4 * i)) & 0x000f000fu) | 0x43004300u;
    const __nv_bfloat162 r = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), bias), s);
    d[i] = *reinterpret_cast<const uint32_t*>(&r);
  }
  __stcs(reinterpret_cast<uint4*>(to), make_uint4(d[0], d[1], d[2], d[3]));
}
__device__ __forceinline__ void w4_unpack8(uint32_t word, __nv_bfloat16 scale, float* to) {
  const float s = __bfloat162float(scale);
  float v[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) v[c] = s * w4_value(word, c);
  __stcs(reinterpret_cast<uint4*>(to), Vec16<float>::pack(v));
  __stcs(reinterpret_cast<uint4*>(to) + 1, Vec16<float>::pack(v + 4));
}

template <typename T, int G>
__global__ void __launch_bounds__(kPackThreads)
w4_unpack_kernel(const uint32_t* __restrict__ codes, const __nv_bfloat16* __restrict__ scales, const PackRows p, T* __restrict__ w) {
  constexpr int LANES = G / 8;
  const int per_row = p.C / 8, lane = threadIdx.x % p.lanes;
  const long long step = (long long)gridDim.x * kPackThreads / p.lanes;
  for (long long row = ((long long)blockIdx.x * kPackThreads + threadIdx.x) / p.lanes; row < p.rows; row += step) {
    const long long e = row / p.N;
    const uint32_t* from = codes + row * per_row;
    const __nv_bfloat16* scale = scales + e * (p.C / G) * p.N + (row - e * p.N);
    T* to = w + row * p.C;
    for (int i0 = lane; i0 < per_row; i0 += p.lanes * kPackUnroll) {
      uint32_t word[kPackUnroll];
      __nv_bfloat16 s[kPackUnroll];
#pragma unroll
      for (int j = 0; j < kPackUnroll; ++j) {
        const int i = i0 + j * p.lanes;
        if (i < per_row) {
          word[j] = __ldcs(from + i);
          s[j] = scale[(size_t)(i / LANES) * p.N];
        }
      }
#pragma unroll
      for (int j = 0; j < kPackUnroll; ++j) {
        const int i = i0 + j * p.lanes;
        if (i < per_row) w4_unpack8(word[j], s[j], to + (size_t)i * 8);
      }
    }
  }
}

static int sm_count_now() {
  int device = 0, sms = 0;
  if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return 0;
  return sms;
}

// Rows and lanes per row (at least a group's); returns the grid, 0 on a CUDA error.
static int pack_rows(int experts, int N, int C, int group, PackRows& p) {
  p.rows = (long long)experts * N;
  p.N = N;
  p.C = C;
  p.lanes = group / 8;
  while (p.lanes < 32 && p.lanes < C / 8) p.lanes *= 2;
  const long long want = (p.rows * p.lanes + kPackThreads - 1) / kPackThreads, most = (long long)sm_count_now() * 8;
  return (int)(want < most ? want : most);
}

template <typename T>
static cudaError_t launch_pack(const void* w, int experts, int N, int C, int group, const moe_w4_t& out, cudaStream_t st) {
  PackRows p;
  const int grid = pack_rows(experts, N, C, group, p);
  if (grid <= 0) return cudaErrorUnknown;
  auto kern = group == 32 ? w4_pack_kernel<T, 32> : group == 64 ? w4_pack_kernel<T, 64> : w4_pack_kernel<T, 128>;
  kern<<<grid, kPackThreads, 0, st>>>((const T*)w, p, (uint32_t*)out.codes, (__nv_bfloat16*)out.scales);
  return cudaGetLastError();
}

template <typename T>
static cudaError_t launch_unpack(const moe_w4_t& w, int experts, int N, int C, int group, void* out, cudaStream_t st) {
  PackRows p;
  const int grid = pack_rows(experts, N, C, group, p);
  if (grid <= 0) return cudaErrorUnknown;
  auto kern = group == 32 ? w4_unpack_kernel<T, 32> : group == 64 ? w4_unpack_kernel<T, 64> : w4_unpack_kernel<T, 128>;
  kern<<<grid, kPackThreads, 0, st>>>((const uint32_t*)w.codes, (const __nv_bfloat16*)w.scales, p, (T*)out);
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
  cudaError_t e = dtype == MOE_DTYPE_FP32 ? launch_pack<float>(d_w, experts, N, C, group, *out, (cudaStream_t)stream)
                                          : launch_pack<__nv_bfloat16>(d_w, experts, N, C, group, *out, (cudaStream_t)stream);
  return e == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

int moe_w4_unpack(int32_t dtype, int32_t experts, int32_t N, int32_t C, int32_t group, const moe_w4_t* w, void* d_out, void* stream) {
  if (dtype != MOE_DTYPE_FP32 && dtype != MOE_DTYPE_BF16) return MOE_ERR_ARG;
  int rc = w4_check(w, experts, N, C, group);
  if (rc != MOE_OK) return rc;
  if (!d_out) return MOE_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(d_out) & 15) return MOE_ERR_ALIGN;
  cudaError_t e = dtype == MOE_DTYPE_FP32 ? launch_unpack<float>(*w, experts, N, C, group, d_out, (cudaStream_t)stream)
                                          : launch_unpack<__nv_bfloat16>(*w, experts, N, C, group, d_out, (cudaStream_t)stream);
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
