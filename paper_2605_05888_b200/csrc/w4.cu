// 4-bit weights with group scales: making them from bf16 or fp32 weights, giving them back, and their products with a few
// rows (moe_w4_pack, moe_w4_unpack, moe_w4_matvec of include/moehub.h).
#include "row_stream.cuh"

namespace moehub {

// ---- packing and unpacking ---------------------------------------------------------------------------------------------------
// A warp takes a segment of a row (rows of few words: several), some words of eight columns per lane in flight: rows,
// segments and matrices are the grid's three dimensions, so that no place has to be divided out and small matrices fill the GPU.  Packing goes
// on to rows further down, whose words are loaded while these are coded; the grid is cut to a few rounds of CTAs for it.
// Measured on 8 bf16 matrices of 14336 x 4096, us, groups of 128 / 64 / 32: unpacking 188 / 193 / 200 (180 / 181 / 183 for the bytes at the copy rate: bound by
// HBM; the smaller the groups, the more scales of two bytes, a row's N apart), packing 218 / 219 / 234: bound by the instructions, about 100 per word (76 % of
// the issue slots; earlier forms: four words per lane in flight and no next ones 280; two, and one round of CTAs 239, 8 rounds 227, 32 rounds 241;
// three CTAs per SM of 8 rounds 245, five 239; two buffers in turn instead of a copy is the present one).  4 fp32 matrices of that size: unpacking
// 214 / 218 / 223, packing 196 / 195 / 196 (162 / 162 / 163 for the bytes): packing has 156 bytes of spills and a word near a border in one of
// twenty steps of a warp, which all its lanes wait for.
constexpr int kPackThreads = 256;
constexpr int kPackUnroll = 2, kUnpackUnroll = 4;  // words per lane
constexpr int kPackCtas = 4, kPackRounds = 8;      // of the packing kernel on an SM

struct PackShape {
  int experts, N, C, lanes;  // lanes: of a row's segment, a power of two
};

typedef unsigned long long f32x2;  // two fp32 numbers for the paired instructions
__device__ __forceinline__ f32x2 pair(float a, float b) {
  f32x2 d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ void unpair(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

template <typename T> struct Eight;  // eight columns
template <> struct Eight<float> {
  uint4 v[2];
  __device__ __forceinline__ void load(const float* p) {
    v[0] = __ldcs(reinterpret_cast<const uint4*>(p));
    v[1] = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
  }
  __device__ __forceinline__ void clear() { v[0] = v[1] = make_uint4(0, 0, 0, 0); }
  // The largest magnitude's bits: an infinity's or a NaN's are larger than any number's.
  __device__ __forceinline__ uint32_t largest() const {
    constexpr uint32_t m = 0x7fffffffu;
    return max(max(max(v[0].x & m, v[0].y & m), max(v[0].z & m, v[0].w & m)), max(max(v[1].x & m, v[1].y & m), max(v[1].z & m, v[1].w & m)));
  }
  __device__ __forceinline__ static uint32_t as_float(uint32_t key) { return key; }
  __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(reinterpret_cast<const uint32_t*>(v)[i]); }
};
template <> struct Eight<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ uint32_t largest() const {
    constexpr uint32_t m = 0x7fff7fffu;
    const uint32_t two = __vmaxu2(__vmaxu2(v.x & m, v.y & m), __vmaxu2(v.z & m, v.w & m));
    return max(two & 0xffffu, two >> 16);
  }
  __device__ __forceinline__ static uint32_t as_float(uint32_t key) { return key << 16; }
  __device__ __forceinline__ float operator[](int i) const {
    const uint32_t w = reinterpret_cast<const uint32_t*>(&v)[i / 2];
    return __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
  }
};

// The code of w without assumptions on s: the nearest integer to w / s, ties to even, within -8..7, plus 8; 8 without a scale.
__device__ __noinline__ uint32_t w4_code(float w, float s) {
  if (!(s > 0.0f)) return 8;
  const double q = rint((double)w / (double)s);
  return (uint32_t)(int)(fmin(fmax(q, -8.0), 7.0) + 8.0);
}
template <typename T>
__device__ __forceinline__ uint32_t w4_word_slow(const Eight<T>& v, float s) {
  uint32_t word = 0;
#pragma unroll
  for (int c = 0; c < 8; ++c) word |= w4_code(v[c], s) << w4_shift(c);
  return word;
}
// A word of codes, for a scale whose inverse is a number.  The quotient is rounded twice: to multiples of 2^-14 (a product with the
// inverse, off by less than 2^-19, and a sum in one step) and then to an integer, ties to even.  The first rounding puts a quotient that is on a border between
// two codes, a multiple of 1/2, there exactly.  Where w is a bf16 number no other comes near one: (2 k + 1) s / 2 has 12
// bits and w 8, so they are equal or 2^-12 of them apart, the quotients 2^-13.  Where w is an fp32 number it may, and |w - k s|, which is exact (k s
// has 12 bits and lies within s of w), is near s / 2 then: such words, a few in a thousand, are done with care.
template <typename T>
__device__ __forceinline__ uint32_t w4_word(const Eight<T>& v, float s) {
  float inverse;
  asm("rcp.approx.f32 %0, %1;" : "=f"(inverse) : "f"(s));
  constexpr float kIntegers = 12582912.0f + 8.0f;  // 1.5 * 2^23: a sum with it is an integer, in the last bits; and the code's 8
  constexpr float kTies = 768.0f;                  // 1.5 * 2^9: a sum with it is a multiple of 2^-14
  const f32x2 inverse2 = pair(inverse, inverse), minus2 = pair(-s, -s), ties2 = pair(kTies, kTies);
  const f32x2 integers2 = pair(kIntegers - kTies, kIntegers - kTies), back2 = pair(-kIntegers, -kIntegers);
  uint32_t word = 0;
  float farthest = 0.0f;
#pragma unroll
  for (int c = 0; c < 8; c += 2) {
    const f32x2 w = pair(v[c], v[c + 1]);
    const f32x2 sum = add2(fma2(w, inverse2, ties2), integers2);
    float a, b;
    unpair(sum, a, b);
    word += __float_as_uint(a) * (1u << w4_shift(c)) + __float_as_uint(b) * (1u << w4_shift(c + 1));
    if (sizeof(T) == 4) {
      float r0, r1;
      unpair(fma2(add2(sum, back2), minus2, w), r0, r1);
      farthest = fmaxf(farthest, fmaxf(fabsf(r0), fabsf(r1)));
    }
  }
  word -= 0x4b400000u * 0x11111111u;  // (the integers' own bits, at every code's place)
  if (sizeof(T) == 4 && farthest > 0.4999f * s) return w4_word_slow(v, s);
  return word;
}

template <typename T, int G>
__global__ void __launch_bounds__(kPackThreads, kPackCtas)
w4_pack_kernel(const T* __restrict__ w, const PackShape p, uint32_t* __restrict__ codes, __nv_bfloat16* __restrict__ scales) {
  constexpr int LANES = G / 8;  // of a group
  const int per_row = p.C / 8, lane = threadIdx.x % p.lanes, rows = kPackThreads / p.lanes;
  const int i0 = blockIdx.y * (p.lanes * kPackUnroll) + lane;
  for (int e = blockIdx.z; e < p.experts; e += gridDim.z) {
    auto load = [&](int n, Eight<T>(&v)[kPackUnroll]) {
#pragma unroll
      for (int j = 0; j < kPackUnroll; ++j) {
        v[j].clear();
        if (n < p.N && i0 + j * p.lanes < per_row) v[j].load(w + ((size_t)e * p.N + n) * p.C + (size_t)(i0 + j * p.lanes) * 8);
      }
    };
    auto code = [&](int n, const Eight<T>(&v)[kPackUnroll]) {
      const size_t row = (size_t)e * p.N + n;
#pragma unroll
      for (int j = 0; j < kPackUnroll; ++j) {
        const int i = i0 + j * p.lanes;
        uint32_t key = v[j].largest();
#pragma unroll
        for (int off = LANES / 2; off > 0; off >>= 1) key = max(key, __shfl_xor_sync(0xffffffffu, key, off));
        if (n >= p.N || i >= per_row) continue;  // (whole groups: per_row is a multiple of LANES)
        const uint32_t bits = Eight<T>::as_float(key);
        const float largest = __uint_as_float(bits);
        __nv_bfloat16 scale;
        uint32_t word;
        if (largest > 1e-28f && bits < 0x7f800000u) {
          constexpr float seventh = 1.0f / 7.0f;  // (the quotient rounded to fp32: a product with the inverse and one correction, Markstein's)
          const float near = largest * seventh;
          scale = __float2bfloat16_rn(__fmaf_rn(__fmaf_rn(-near, 7.0f, largest), seventh, near));
          word = w4_word(v[j], __bfloat162float(scale));
        } else {  // zeros, tiny numbers; a NaN or an infinity: NaN
          scale = __float2bfloat16_rn(bits < 0x7f800000u ? __fdiv_rn(largest, 7.0f) : __int_as_float(0x7fc00000));
          word = w4_word_slow(v[j], __bfloat162float(scale));
        }
        __stcs(codes + row * per_row + i, word);
        if (i % LANES == 0) scales[((size_t)e * (p.C / G) + i / LANES) * p.N + n] = scale;
      }
    };
    Eight<T> v[kPackUnroll], next[kPackUnroll];  // (in turn)
    const int step = gridDim.x * rows;
    int n = blockIdx.x * rows + threadIdx.x / p.lanes, left = p.N - blockIdx.x * rows;
    load(n, v);
    while (true) {
      if (left > step) load(n + step, next);
      code(n, v);
      if (left <= step) break;
      if (left - step > step) load(n + 2 * step, v);
      code(n + step, next);
      if (left - step <= step) break;
      left -= 2 * step;
      n += 2 * step;
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
w4_unpack_kernel(const uint32_t* __restrict__ codes, const __nv_bfloat16* __restrict__ scales, const PackShape p, T* __restrict__ w) {
  constexpr int LANES = G / 8;
  const int per_row = p.C / 8, lane = threadIdx.x % p.lanes;
  const int n = blockIdx.x * (kPackThreads / p.lanes) + threadIdx.x / p.lanes;
  const int i0 = blockIdx.y * (p.lanes * kUnpackUnroll) + lane;
  if (n >= p.N) return;
  for (int e = blockIdx.z; e < p.experts; e += gridDim.z) {
    const size_t row = (size_t)e * p.N + n;
    uint32_t word[kUnpackUnroll];
    __nv_bfloat16 s[kUnpackUnroll];
#pragma unroll
    for (int j = 0; j < kUnpackUnroll; ++j) {
      const int i = i0 + j * p.lanes;
      if (i < per_row) {
        word[j] = __ldcs(codes + row * per_row + i);
        s[j] = scales[((size_t)e * (p.C / G) + i / LANES) * p.N + n];
      }
    }
#pragma unroll
    for (int j = 0; j < kUnpackUnroll; ++j) {
      const int i = i0 + j * p.lanes;
      if (i < per_row) w4_unpack8(word[j], s[j], w + row * p.C + (size_t)i * 8);
    }
  }
}

static int sm_count_now() {
  int device = 0, sms = 0;
  if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return 0;
  return sms;
}

// The grid, and the lanes of a row's segment: at least a group's, up to a warp's, more where a row would have more segments than a grid's
// second dimension may count (rows of 2^25 columns).
static dim3 pack_grid(PackShape& p, int group, int unroll) {
  p.lanes = group / 8;
  while ((p.lanes < 32 && p.lanes < p.C / 8) || (p.lanes < kPackThreads && p.C / 8 > 65535 * p.lanes * unroll)) p.lanes *= 2;
  const int rows = kPackThreads / p.lanes, words = p.lanes * unroll;
  return dim3((p.N + rows - 1) / rows, (p.C / 8 + words - 1) / words, p.experts < 65535 ? p.experts : 65535);
}

template <typename T>
static cudaError_t launch_pack(const void* w, PackShape p, int group, const moe_w4_t& out, cudaStream_t st) {
  dim3 grid = pack_grid(p, group, kPackUnroll);
  const int sms = sm_count_now();
  if (sms <= 0) return cudaErrorUnknown;
  grid.x = min(grid.x, max(1u, (unsigned)(sms * kPackCtas * kPackRounds) / (grid.y * grid.z)));
  auto kern = group == 32 ? w4_pack_kernel<T, 32> : group == 64 ? w4_pack_kernel<T, 64> : w4_pack_kernel<T, 128>;
  kern<<<grid, kPackThreads, 0, st>>>((const T*)w, p, (uint32_t*)out.codes, (__nv_bfloat16*)out.scales);
  return cudaGetLastError();
}

template <typename T>
static cudaError_t launch_unpack(const moe_w4_t& w, PackShape p, int group, void* out, cudaStream_t st) {
  const dim3 grid = pack_grid(p, group, kUnpackUnroll);
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
template <int G, int NT, bool SMALL>
__global__ void __launch_bounds__(RsSizes<W4<G, SMALL>, NT>::THREADS, 1)
w4_matvec_kernel(const __grid_constant__ W4MatvecParams p, int batch) {
  typedef RsSizes<W4<G, SMALL>, NT> Z;
  constexpr int SLOTS = 8 * NT;
  extern __shared__ __align__(128) unsigned char dynamic[];
  __shared__ unsigned short used[32];
  __shared__ unsigned char count[32], token[32 * SLOTS];
  __shared__ int entries;
  float* slots = reinterpret_cast<float*>(dynamic + Z::RING);
  const uint32_t ring = smem_u32(dynamic) + threadIdx.x / 32 * Z::WARP_RING;
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
    const RsList list{used, count, token, nullptr, entries};
    const RsOperand op{p.codes, p.codes, p.scales, p.scales, p.x + (size_t)m0 * p.C, 0, p.N, p.C, p.experts, 0};
    typedef RowStream<W4<G, SMALL>, NT, kRsRows> Stream;
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
    rs.run(nullptr, slots, [](int, int, int&) { return 0.0f; }, finish);
    __syncthreads();
    rs.join(slots, finish);
    __syncthreads();
  }
}

template <int G, int NT, bool SMALL>
static cudaError_t launch_matvec(const W4MatvecParams& q, int device, int sms, cudaStream_t st) {
  typedef RsSizes<W4<G, SMALL>, NT> Z;
  static SmemAttrOnce once;
  cudaError_t e = ensure_dynamic_smem(w4_matvec_kernel<G, NT, SMALL>, Z::BYTES, device, once);
  if (e != cudaSuccess) return e;
  w4_matvec_kernel<G, NT, SMALL><<<sms, Z::THREADS, Z::BYTES, st>>>(q, q.experts > 1 ? 32 : 8 * NT);
  return cudaGetLastError();
}

// 16 rows of one matrix at a time (with eight warps, for the registers) where there are more than eight: groups of 128, 7168 x 7168, us, by
// eights / by sixteens: 8 rows 12.0 / 15.0, 9 rows 22.0 / 15.5, 32 rows 43.1 / 30.4, 48 rows 63.5 / 45.1 (4.1 for the bytes: every sixteen rows read and expand
// them anew); of several matrices rows that share one are few (24 rows of 60 matrices of 2817 x 2048 26.8 / 32.3).  The small code where a CTA has no
// more than sixteen rows of the matrices: 1408 x 2048, small / other, 4.9 / 5.3, 16 rows 6.1 / 6.5; 7168 x 7168 16 rows 19.0 / 18.1; 24 rows of 60
// matrices 27.2 / 26.9.
template <int G>
static cudaError_t launch_matvec(const W4MatvecParams& q, cudaStream_t st) {
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const int sms = sm_count_now();
  if (sms <= 0) return cudaErrorUnknown;
  const bool small = (long long)q.N * (q.experts > 1 ? min(q.M, 32) : 1) <= 16ll * sms;
  if (q.M <= 8 || q.experts > 1) return small ? launch_matvec<G, 1, true>(q, device, sms, st) : launch_matvec<G, 1, false>(q, device, sms, st);
  return small ? launch_matvec<G, 2, true>(q, device, sms, st) : launch_matvec<G, 2, false>(q, device, sms, st);
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
  cudaError_t e = dtype == MOE_DTYPE_FP32 ? launch_pack<float>(d_w, PackShape{experts, N, C, 0}, group, *out, (cudaStream_t)stream)
                                          : launch_pack<__nv_bfloat16>(d_w, PackShape{experts, N, C, 0}, group, *out, (cudaStream_t)stream);
  return e == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

int moe_w4_unpack(int32_t dtype, int32_t experts, int32_t N, int32_t C, int32_t group, const moe_w4_t* w, void* d_out, void* stream) {
  if (dtype != MOE_DTYPE_FP32 && dtype != MOE_DTYPE_BF16) return MOE_ERR_ARG;
  int rc = w4_check(w, experts, N, C, group);
  if (rc != MOE_OK) return rc;
  if (!d_out) return MOE_ERR_ARG;
  if (reinterpret_cast<uintptr_t>(d_out) & 15) return MOE_ERR_ALIGN;
  cudaError_t e = dtype == MOE_DTYPE_FP32 ? launch_unpack<float>(*w, PackShape{experts, N, C, 0}, group, d_out, (cudaStream_t)stream)
                                          : launch_unpack<__nv_bfloat16>(*w, PackShape{experts, N, C, 0}, group, d_out, (cudaStream_t)stream);
  return e == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

int moe_w4_matvec(int32_t experts, int32_t N, int32_t C, int32_t group, const moe_w4_t* w, int32_t M, const void* d_x,
                  const int32_t* d_expert, void* d_y, void* stream) {
  int rc = w4_check(w, experts, N, C, group);
  if (rc != MOE_OK) return rc;
  if (M < 0) return MOE_ERR_ARG;
  if (M == 0) return MOE_OK;
  if (!d_x || !d_y || (experts > 1 && !d_expert)) return MOE_ERR_ARG;
  if (experts > 65535 || N > (1 << 25) || M > (1 << 30)) return MOE_ERR_UNSUPPORTED;  // (matrix numbers are held in 16 bits, numbers of rows in 32)
  if (((reinterpret_cast<uintptr_t>(d_x) | reinterpret_cast<uintptr_t>(d_y)) & 15) || (reinterpret_cast<uintptr_t>(d_expert) & 3))
    return MOE_ERR_ALIGN;
  if (d_x == d_y) return MOE_ERR_ARG;  // (rows are read while others' results are written)
  const W4MatvecParams q{w->codes, (const __nv_bfloat16*)w->scales, (const __nv_bfloat16*)d_x, d_expert, (__nv_bfloat16*)d_y, experts, N, C, M};
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = group == 32 ? launch_matvec<32>(q, st) : group == 64 ? launch_matvec<64>(q, st) : launch_matvec<128>(q, st);
  return e == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

}  // extern "C"
