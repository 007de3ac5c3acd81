// The whole MoE layer (paper Section II-A, steps 1-5) for a few tokens in one launch, on bf16, fp32 or 4-bit expert weights
// (moe_layer_few, moe_layer_few_w4 of include/moehub.h).
//
// As many CTAs as SMs, all resident (a cooperative launch), go through three parts with grid-wide barriers between them (1.2 us each;
// a third one where CTAs share outputs):
//   router   every CTA forms the logits of a few experts, or of slices of them where there are few experts
//   gate/up  every CTA selects the picks for itself from the logits, and computes its share of the rows
//            S[u, t, f] = silu(x_t Wg[e_u, f]) * (x_t Wu[e_u, f]) of the used experts e_0 < e_1 < ...
//   down     every CTA computes its share of the outputs y[t, h] = sum_u w[u, t] sum_f S[u, t, f] Wd[e_u, h, f]: all the used
//            experts' columns of a row are in one CTA, so there is no separate combine step
// No row is copied, and no table is built that only a later launch would read.  The weights go through row_stream.cuh.
//
// Bound by reading the picked experts' weights once; for one token of small experts by latencies, which the trace of one Qwen-like token shows,
// us: launch and router 2.4, barrier 1.2 of it, selection 2, gate/up 7 (46 MB), joins 1, the others' arrival and the barrier 3, down 4 (23 MB), end 1.
// Measured, device time by graph replay, us, moe_layer (three launches or more) / this / the picked experts' bytes at the copy rate (which a stream
// that only reads can beat by some per cent).  bf16: Qwen-like 1 token 27.4 / 21.8 / 10.5, 16 tokens 129 / 118 / 104; Mixtral-like 1 token
// 123 / 111 / 107, 5 tokens 378 / 335 / 340, 16 tokens 462 / 430 / 429; DeepSeek-like 1 token 145 / 114 / 107, 16 tokens 1279 / 1193 / 1252; of 8
// experts of 512 x 512, 4 tokens, 13.8 / 14.1 / 1.4 (latencies alone).  fp32: 16 experts of 1020 x 2044, 3 tokens, 105 / 37 / 23; Phi-like 8 tokens
// 724 / 487 / 479.  4 bits (this / expected bytes), groups of 128: Qwen-like 1 token 18.1 / 2.8, Mixtral-like 1 token 57 / 28, 7 tokens 171 / 95 (all
// eight experts: 116), DeepSeek-like 16 tokens 525 / 350; groups of 64 and 32: Mixtral-like 7 tokens 182 / 98 and 203 / 104.  No unit and not HBM is full
// there: instructions that unpack the codes, and their latencies (row_stream.cuh).
#include "route_common.cuh"
#include "row_stream.cuh"

namespace moehub {

constexpr int kLfMaxWarps = 16;
constexpr int kLfTokens = MOE_FEW_MAX_TOKENS;
constexpr int kLfPicks = 32;  // most picks per token

struct LfMatrix {
  const void* w;                // [E, N, C] of the weights' type, or the codes
  const __nv_bfloat16* scales;  // [E, C / group, N] (4 bits)
};

struct LayerFewParams {
  const void* x;
  const void* wr;
  const float* bias;
  LfMatrix wg, wu, wd;
  void* y;
  int T, H, E, K, F, renorm, tp;
  int slices, slice_cols;  // of the router's sums
  float* logits;           // [slices, T, E]
  void* inter;             // the gate / up results of the entries' tokens, [entries, 8, F], on tensor cores followed by what rounding them left
  unsigned* sync;          // three barriers' counters, 128 bytes apart
  float* partial;          // (split) [parts, T, H]: the outputs' parts, as many as CTAs have some of a tile
  int split;               // of the outputs, see RsOperand
  int* topk_idx;           // the picks and rows per expert, as moe_layer leaves them (every TP shard listed)
  float* topk_w;
  int* expert_count;
  int* status;
  unsigned long long wait_ns;
};

// Every CTA of the grid arrives exactly once per launch and barrier, also one whose wait ran out before: together they add 2^31, so
// that the counter's highest bit flips with the last one and what is below it is as it was.  What was written before arrive() is
// visible behind wait() (to loads that miss L1); arrive()'s result (of thread 0) is for wait().  late: the wait ran out (thread 0's).
__device__ __forceinline__ unsigned grid_arrive(const LayerFewParams& p, int which) {
  __syncthreads();
  unsigned before = 0;
  if (threadIdx.x == 0) {
    const unsigned mine = blockIdx.x == 0 ? 0x80000000u - (gridDim.x - 1) : 1u;
    asm volatile("atom.add.release.gpu.global.u32 %0, [%1], %2;" : "=r"(before) : "l"(p.sync + 32 * which), "r"(mine) : "memory");
  }
  return before;
}
__device__ __forceinline__ void grid_wait(const LayerFewParams& p, int which, unsigned before, bool& late) {
  if (threadIdx.x == 0) {
    unsigned long long t0 = 0;
    while (!((before ^ (unsigned)ld_acquire(reinterpret_cast<int*>(p.sync + 32 * which))) >> 31)) {
      const unsigned long long now = globaltimer();
      if (t0 == 0) t0 = now;
      if (now - t0 > p.wait_ns) {
        late = true;
        set_status(p.status, MOE_ERR_TIMEOUT, kWaitGrid);
        break;
      }
    }
  }
  __syncthreads();
}
__device__ __forceinline__ void grid_barrier(const LayerFewParams& p, int which, bool& late) { grid_wait(p, which, grid_arrive(p, which), late); }

// Entries (see RsList): of the gate / up product one per used expert and eight tokens of it, of the down product one per expert and
// `FEW` of them (four or eight on tensor cores).  Most there can be: 256 experts, and one more per eight (four) of the remaining 256 of
// sixteen times 32 picks.
constexpr int kLfSlots = 8, kLfEntries = 288, kLfDownEntries = 320;
struct LfShared {
  float w[kLfTokens * kLfPicks];                    // the picks' weights
  unsigned short used[kLfEntries];                  // an entry's expert, ascending
  unsigned char count[kLfEntries];
  unsigned char token[kLfEntries * kLfSlots];       // its tokens
  unsigned char pick[kLfEntries * kLfSlots];        // and which of a token's picks it is
  unsigned short down_used[kLfDownEntries], down_row[kLfDownEntries];  // row: of the results, eight per gate / up entry
  unsigned char down_count[kLfDownEntries];
};
constexpr int kLfBatch = 2;  // experts that a CTA scores at a time
struct LfSelect {            // where the rows are streamed through later
  float red[kLfMaxWarps][kLfBatch * kLfTokens];
  int idx[kLfTokens * kLfPicks];
  unsigned mask[kMaxExperts];            // the tokens that picked an expert
  unsigned used[kMaxExperts / 32];       // bit per expert: picked at all,
  unsigned many[3][kMaxExperts / 32];    // by more than 4, 8, 12 tokens
};

template <int N>
__device__ __forceinline__ float lf_dot(const uint4& x, const uint4& w);
template <>
__device__ __forceinline__ float lf_dot<4>(const uint4& x, const uint4& w) {
  float a[4], b[4], s = 0.0f;
  Vec16<float>::unpack(x, a);
  Vec16<float>::unpack(w, b);
#pragma unroll
  for (int j = 0; j < 4; ++j) s = __fmaf_rn(a[j], b[j], s);
  return s;
}
template <>
__device__ __forceinline__ float lf_dot<8>(const uint4& x, const uint4& w) {
  const uint32_t a[4] = {x.x, x.y, x.z, x.w}, b[4] = {w.x, w.y, w.z, w.w};
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) s = fma_bf16_hi(a[j], b[j], fma_bf16_lo(a[j], b[j], s));
  return s;
}

// The logits (or a slice's part of them): a CTA takes kLfBatch experts of a slice, columns over its threads.  TT: tokens at most.
template <typename T, int TT>
__device__ __forceinline__ void lf_router(const LayerFewParams& p, LfSelect& s) {
  constexpr int N = Vec16<T>::N, SUMS = kLfBatch * TT;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int batches = (p.E + kLfBatch - 1) / kLfBatch;
  for (int task = blockIdx.x; task < batches * p.slices; task += gridDim.x) {
    const int slice = task / batches, e0 = (task - slice * batches) * kLfBatch;
    const int c0 = slice * p.slice_cols, c1 = min(p.H, c0 + p.slice_cols);
    float acc[SUMS] = {};
    for (int c = c0 + (int)threadIdx.x * N; c < c1; c += blockDim.x * N) {
      uint4 w[kLfBatch];
#pragma unroll
      for (int i = 0; i < kLfBatch; ++i) w[i] = __ldg(reinterpret_cast<const uint4*>((const T*)p.wr + (size_t)min(e0 + i, p.E - 1) * p.H + c));
      constexpr int TG = TT < 8 ? TT : 8;  // tokens whose loads are in flight together (past the last one: the last one's again)
#pragma unroll
      for (int t0 = 0; t0 < TT; t0 += TG) {
        uint4 x[TG];
#pragma unroll
        for (int t = 0; t < TG; ++t) x[t] = __ldg(reinterpret_cast<const uint4*>((const T*)p.x + (size_t)min(t0 + t, p.T - 1) * p.H + c));
#pragma unroll
        for (int t = 0; t < TG; ++t)
#pragma unroll
          for (int i = 0; i < kLfBatch; ++i) acc[i * TT + t0 + t] += lf_dot<N>(x[t], w[i]);
      }
    }
    // Sums over the lanes: each step halves the values a lane holds, so that SUMS of them take SUMS - 1 exchanges.
    int mine = 0;
#pragma unroll
    for (int step = 0; step < 5; ++step) {
      const int off = 16 >> step, n = (SUMS / 2) >> step;
      if (n >= 1) {
        const bool upper = lane & off;
#pragma unroll
        for (int j = 0; j < SUMS / 2; ++j) {
          if (j >= n) break;
          const float keep = upper ? acc[j + n] : acc[j], give = upper ? acc[j] : acc[j + n];
          acc[j] = keep + __shfl_xor_sync(0xffffffffu, give, off);
        }
        mine += upper ? n : 0;
      } else {
        acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], off);
      }
    }
    if (lane % (32 / SUMS) == 0) s.red[warp][mine] = acc[0];
    __syncthreads();
    if ((int)threadIdx.x < SUMS) {
      float sum = 0.0f;
      for (int i = 0; i < (int)blockDim.x / 32; ++i) sum += s.red[i][threadIdx.x];
      const int e = e0 + (int)threadIdx.x / TT, t = threadIdx.x % TT;
      if (e < p.E && t < p.T) __stcg(p.logits + ((size_t)slice * p.T + t) * p.E + e, sum);
    }
    __syncthreads();
  }
}

// A warp selects the picks of token t (as select_topk does, from registers).
template <int NJ>
__device__ __forceinline__ void lf_pick(const LayerFewParams& p, LfShared& s, LfSelect& q, int t) {
  const int lane = threadIdx.x % 32;
  float v[NJ] = {}, b[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) b[j] = p.bias != nullptr && lane + 32 * j < p.E ? __ldg(p.bias + lane + 32 * j) : 0.0f;
  const float* from = p.logits + t * p.E + lane;
  for (int i0 = 0; i0 < p.slices; i0 += 4) {  // four slices' loads in flight
    float l[4][NJ];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) l[i][j] = i0 + i < p.slices && lane + 32 * j < p.E ? __ldcg(from + (i0 + i) * p.T * p.E + 32 * j) : 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) v[j] += l[i][j];
  }
  unsigned key[NJ];  // 0: no expert, or picked already
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int e = lane + 32 * j;
    v[j] += b[j];
    key[j] = e < p.E ? max(order_key(v[j]), 1u) : 0u;
  }
  unsigned my_key = 0, first_key = 0;
  int my_e = 0;
  for (int k = 0; k < p.K; ++k) {
    unsigned best = key[0];
#pragma unroll
    for (int j = 1; j < NJ; ++j) best = max(best, key[j]);
    best = __reduce_max_sync(0xffffffffu, best);
    unsigned e = 0xffffffffu;
#pragma unroll
    for (int j = NJ - 1; j >= 0; --j)
      if (key[j] == best) e = (unsigned)(lane + 32 * j);
    e = __reduce_min_sync(0xffffffffu, e);
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if (e == (unsigned)(lane + 32 * j)) key[j] = 0u;
    if (k == 0) first_key = best;
    if (lane == k) { my_e = (int)e; my_key = best; }
  }
  auto value = [](unsigned k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); };
  const float m = value(first_key);
  float z = 0.0f;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
    if (lane + 32 * j < p.E) z += expf(v[j] - m);
  z = group_sum<32>(z);
  float w = lane < p.K ? expf(value(my_key) - m) / z : 0.0f;
  if (p.renorm) w = w / group_sum<32>(w);
  if (lane < p.K) {
    s.w[t * p.K + lane] = w;
    q.idx[t * p.K + lane] = my_e;
    atomicOr(&q.mask[my_e], 1u << t);
    atomicOr(&q.used[my_e / 32], 1u << (my_e % 32));
    if (blockIdx.x == 0)
      for (int sh = 0; sh < p.tp; ++sh) {
        p.topk_idx[(t * p.K + lane) * p.tp + sh] = my_e * p.tp + sh;
        p.topk_w[(t * p.K + lane) * p.tp + sh] = w;
      }
  }
}

// Before the barrier.
__device__ __forceinline__ void lf_clear(LfSelect& q) {
  if (threadIdx.x < kMaxExperts) q.mask[threadIdx.x] = 0;
  if (threadIdx.x < kMaxExperts / 32) q.used[threadIdx.x] = q.many[0][threadIdx.x] = q.many[1][threadIdx.x] = q.many[2][threadIdx.x] = 0;
}

// Every CTA selects for itself; n, n_down: the numbers of entries.  FEW: most tokens of one of the down product, 4 or 8.
template <int FEW>
__device__ __forceinline__ void lf_select(const LayerFewParams& p, LfShared& s, LfSelect& q, int& n, int& n_down) {
  const int tid = threadIdx.x;
  for (int t = tid / 32; t < p.T; t += blockDim.x / 32) {
    if (p.E <= 64) lf_pick<2>(p, s, q, t);
    else lf_pick<8>(p, s, q, t);
  }
  __syncthreads();
  if (p.T > 4) {
    if (tid < kMaxExperts)
      for (int i = 0; i < 3; ++i)
        if (__popc(q.mask[tid]) > 4 * (i + 1)) atomicOr(&q.many[i][tid / 32], 1u << (tid % 32));
    __syncthreads();
  }
  n = n_down = 0;
#pragma unroll
  for (int i = 0; i < kMaxExperts / 32; ++i) {
    const int used = __popc(q.used[i]), many = __popc(q.many[1][i]);
    n += used + many;
    n_down += used + many + (FEW == 4 ? __popc(q.many[0][i]) + __popc(q.many[2][i]) : 0);
  }
  for (int a = tid; a < p.T * p.K; a += blockDim.x) {
    const int t = a / p.K, e = q.idx[a];
    int at = 0, down = 0;  // entries of the experts before e
#pragma unroll
    for (int i = 0; i < kMaxExperts / 32; ++i) {
      const unsigned below = i < e / 32 ? 0xffffffffu : i == e / 32 ? (1u << (e % 32)) - 1u : 0u;
      const int both = __popc(q.used[i] & below) + __popc(q.many[1][i] & below);
      at += both;
      down += both + (FEW == 4 ? __popc(q.many[0][i] & below) + __popc(q.many[2][i] & below) : 0);
    }
    const int rank = __popc(q.mask[e] & ((1u << t) - 1u)), tokens = __popc(q.mask[e]);
    at += rank / kLfSlots;
    down += rank / FEW;
    s.token[at * kLfSlots + rank % kLfSlots] = (unsigned char)t;
    s.pick[at * kLfSlots + rank % kLfSlots] = (unsigned char)(a - t * p.K);
    if (rank % kLfSlots == 0) {
      s.used[at] = (unsigned short)e;
      s.count[at] = (unsigned char)min(kLfSlots, tokens - rank);
    }
    if (rank % FEW == 0) {
      s.down_used[down] = (unsigned short)e;
      s.down_row[down] = (unsigned short)(at * kLfSlots + rank % kLfSlots);
      s.down_count[down] = (unsigned char)min(FEW, tokens - rank);
    }
  }
  if (blockIdx.x == 0)
    for (int e = tid; e < p.E * p.tp; e += blockDim.x) p.expert_count[e] = __popc(q.mask[e / p.tp]);
  __syncthreads();
}

__device__ __forceinline__ float lf_silu_mul(float g, float u) { return g / (1.0f + expf(-g)) * u; }

// DOWN: eights of token slots in the down product's entries, so that these have up to 4 * DOWN tokens as two numbers each.  2 where an expert
// has at least two of more than four tokens on average (launch below): its entries of more than four tokens else read its down rows twice,
// the second time from L2.  Measured, us, 1 / 2: Mixtral-like 16 tokens 477 / 429, 11 tokens 435 / 427, 8 tokens 403 / 406, 6 tokens 387 / 389,
// Phi-like 16 tokens 331 / 326, 8 tokens 242.6 / 244.4, Qwen-like 6 tokens 65.9 / 67.4.
template <typename W, int DOWN>
__global__ void __launch_bounds__(RsSizes<W, 1>::THREADS, 1)
layer_few_kernel(const __grid_constant__ LayerFewParams p) {
  typedef typename RsFormat<W>::X X;
  typedef RsSizes<W, 1> Z;
  extern __shared__ __align__(128) unsigned char dynamic[];
  __shared__ LfShared s;
  static_assert(sizeof(LfSelect) <= Z::RING && Z::WARPS <= kLfMaxWarps && Z::THREADS >= kMaxExperts, "the selection's tables lie in the ring");
  LfSelect& q = *reinterpret_cast<LfSelect*>(dynamic);
  float* slots = reinterpret_cast<float*>(dynamic + Z::RING);
  const uint32_t ring = smem_u32(dynamic) + threadIdx.x / 32 * Z::WARP_RING;
  const int lane = threadIdx.x % 32;
  if (blockIdx.x == 0 && threadIdx.x == 0) p.status[0] = p.status[1] = 0;
  if (p.T <= 1) lf_router<X, 1>(p, q);
  else if (p.T <= 4) lf_router<X, 4>(p, q);
  else if (p.T <= 8) lf_router<X, 8>(p, q);
  else lf_router<X, kLfTokens>(p, q);
  lf_clear(q);
  bool late = false;
  grid_barrier(p, 0, late);
  int entries, down_entries;
  lf_select<sizeof(X) == 2 ? 4 * DOWN : kLfSlots>(p, s, q, entries, down_entries);
  const RsList list{s.used, s.count, s.token, nullptr, entries}, down_list{s.down_used, s.down_count, nullptr, s.down_row, down_entries};

  // gate and up rows of the used experts
  const long long rest = (long long)entries * kLfSlots * p.F;
  const RsOperand gate_up{p.wg.w, p.wu.w, p.wg.scales, p.wu.scales, p.x, 0, p.F, p.H, p.E, 0};
  typedef RowStream<W, 1, kRsPairs> Up;
  Up up(gate_up, list, ring);
  auto finish_up = [&](int u, int row, int n0, int, const float*) {
#pragma unroll
    for (int j = 0; j < Z::REGS; ++j) {
      if (Up::kMma && j % 4 >= 2) continue;
      const float upper = Up::kMma ? up.acc[Up::kMma ? j + 2 : j] : __shfl_down_sync(0xffffffffu, up.acc[j], kRsRun);
      const int t = up.token(j), f = up.row_of(j);
      if (t < s.count[u] && f < n0 && (Up::kMma || lane < kRsRun)) {
        const float v = lf_silu_mul(up.acc[j], upper);
        X* to = (X*)p.inter + ((size_t)u * kLfSlots + t) * p.F + row + f;
        if (Up::kMma) {
          float near = to_float(from_float<X>(v));
          if (fabsf(near) == INFINITY && fabsf(v) < INFINITY) near = __uint_as_float(__float_as_uint(v) & 0xffff0000u);  // (a number yet)
          to[0] = from_float<X>(near);
          to[rest] = from_float<X>(fabsf(near) < INFINITY ? v - near : 0.0f);
        } else {
          to[0] = from_float<X>(v);
        }
      }
    }
  };
  up.run(nullptr, slots, [](int, int, int&) { return 0.0f; }, finish_up);

  __syncthreads();
  up.join(slots, finish_up);
  const unsigned arrived = grid_arrive(p, 1);

  // the outputs; the first down rows are on their way while the other CTAs finish
  const RsOperand down_op{p.wd.w, p.wd.w, p.wd.scales, p.wd.scales, p.inter, rest, p.H, p.F, p.E, p.split};
  typedef RowStream<W, DOWN, kRsSum> Down;
  static_assert(RsSizes<W, DOWN>::WARP_RING == Z::WARP_RING && RsSizes<W, DOWN>::WARPS == Z::WARPS, "the ring is the same");
  Down down(down_op, down_list, ring);
  Down start = down;
  down.prefetch();
  grid_wait(p, 1, arrived, late);
  auto store = [&](int row, int t, float v, int part) {
    const size_t at = (size_t)t * p.H + row;
    if (p.split) p.partial[(size_t)part * p.T * p.H + at] = v;
    else ((X*)p.y)[at] = from_float<X>(v);
  };
  auto finish_down = [&](int, int row, int n0, int n1, const float* sums) {
    const int r = lane % kRsRun;
    if (r < (lane < kRsRun ? n0 : n1))
      for (int t = 0; t < p.T; ++t) store(row + (lane < kRsRun ? 0 : n0) + r, t, sums[Down::sum_at(t, lane)], 0);
  };
  auto weight = [&](int u, int t, int& token) {
    const int at = s.down_row[u] + t;
    token = s.token[at];
    return s.w[token * p.K + s.pick[at]];
  };
  down.run(&start, slots, weight, finish_down);
  __syncthreads();
  down.join_sums(slots, p.T, store);
  if (p.split) {
    grid_barrier(p, 2, late);
    for (int i = blockIdx.x * Z::THREADS + threadIdx.x; i < p.T * p.H; i += gridDim.x * Z::THREADS)
      ((X*)p.y)[i] = from_float<X>(down.combine(p.partial + i, (size_t)p.T * p.H, (unsigned)i % (unsigned)p.H));
  }
  if (late) set_status(p.status, MOE_ERR_TIMEOUT, kWaitGrid);  // (once more: CTA 0 may have begun, and cleared it, after this one gave up)
}

template <typename W, int DOWN = 1>
static cudaError_t launch_cooperative(const moe_plan* p, const LayerFewParams& q, cudaStream_t st) {
  static SmemAttrOnce once;
  auto kern = layer_few_kernel<W, DOWN>;
  cudaError_t e = ensure_dynamic_smem(kern, RsSizes<W, 1>::BYTES, p->device, once);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p->sm_count);
  cfg.blockDim = dim3(RsSizes<W, 1>::THREADS);
  cfg.dynamicSmemBytes = RsSizes<W, 1>::BYTES;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, q);
}
// Reading one product's rows of as many experts as the tokens can pick, at 6 TB/s.
static double reading_us(const moe_plan* p, int group) {
  const moe_config_t& c = p->cfg;
  const double bits = group > 0 ? 4.0 + 16.0 / group : c.dtype == MOE_DTYPE_BF16 ? 16.0 : 32.0;
  return (double)min(c.T * p->route_K, p->route_E) * c.H * c.F * p->tp * bits / 8.0 / 6.0e6;
}
// (4 bits) Below this the small form of the code.  Measured, us, small / other: Qwen-like 1 token 18.4 / 19.8, 4 tokens (4 us of reading) 35.6 / 39.4,
// 16 tokens (15 us) 66.7 / 67.6, 16 tokens of 64 experts of 1024 x 1024, top-4 (6 us) 41.0 / 39.8, Mixtral-like 1 token (10 us) 60.3 / 57.8, 7 tokens (40 us)
// 181 / 171, DeepSeek-like 1 token (10 us) 67.7 / 63.8, 4 tokens (40 us) 189 / 179, 16 tokens 559 / 547.
constexpr double kSmallUs = 9.0;

// Whether all CTAs share all outputs' terms, which costs a third barrier and the joining of the parts, 3 to 4 us, and saves what a CTA with
// rows of its own loses: with 4 bits, which are bound by instructions, to the rows that its sixteens lack (48.4 rows take as long as 64) and to
// warps' last units; else, where it has fewer than sixteen rows, to loops over many columns that are bound by latencies.  Measured, whole
// layers, us, rows of its own / shared.  4 bits: DeepSeek-like 1 token 63.7 / 66.5, 2 tokens 105.8 / 105.1, 4 tokens 189 / 179, 16 tokens 583 / 529; Mixtral-like
// 1 token 57.8 / 62.0, 7 tokens 174 / 171; Qwen-like 1 token 18.4 / 21.5, 4 tokens 35.8 / 38.2, 16 tokens 78.5 / 66.8.  16 tokens, 64 experts of 1024 x 1024,
// top-4: 4 bits 47 / 41, bf16 69 / 57, fp32 137 / 101; 1 token, 16 of 1024 x 2048: bf16 15.2 / 16.0, fp32 21.2 / 21.8, 3 tokens 26.4 / 26.6 and 40.7 / 34.6.
static bool split_outputs(const moe_plan* p, int group) {
  const moe_config_t& c = p->cfg;
  const int G = p->sm_count, picked = min(c.T * p->route_K, p->route_E), F = c.F * p->tp, all_tiles = (c.H + kRsTile - 1) / kRsTile;
  if ((long long)all_tiles * kLfDownEntries * ((F + 31) / 32) >= 1ll << 31) return false;  // (numbers of units)
  const double us = reading_us(p, group);
  if (group == 0) return us * ((double)G * kRsRun / c.H - 1.0) > 4.5;
  // a warp's units of sixteen rows, alone and shared; the multiplication is taken to last twice as long as the reading (1.5 to 2 times)
  const int rows = (c.H + G - 1) / G, tiles = (rows + kRsTile - 1) / kRsTile, runs = (rows + tiles - 1) / tiles > kRsRun || us >= kSmallUs ? 2 : 1;
  const long long units = (long long)picked * ((F + RsFormat<W4<32, false>>::COLS - 1) / RsFormat<W4<32, false>>::COLS), warps = RsFormat<W4<32, false>>::WARPS;
  const double alone = (double)((tiles * units + warps - 1) / warps * runs), shared = (double)((all_tiles * units + warps * G - 1) / (warps * G) * 2);
  return 2.0 * us * (alone / shared - 1.0) > 4.5;
}

// A plan's first launch is ordered behind what plan creation did on the default stream, which the call's own stream may not follow: on the
// device, or where that is being captured on the host (a graph cannot wait for what is not part of it; the mode allows a wait in a capture).
static cudaError_t few_start(moe_plan* p, cudaStream_t st) {
  if (p->few_ready == nullptr) return cudaSuccess;
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  cudaError_t e = cudaStreamIsCapturing(st, &capture);
  if (e != cudaSuccess) return e;
  if (capture == cudaStreamCaptureStatusNone) {
    e = cudaStreamWaitEvent(st, p->few_ready, 0);
  } else {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    cudaThreadExchangeStreamCaptureMode(&mode);
    e = cudaEventSynchronize(p->few_ready);
    cudaThreadExchangeStreamCaptureMode(&mode);
  }
  if (e != cudaSuccess) return e;
  cudaEventDestroy(p->few_ready);  // (what waits for it does so all the same)
  p->few_ready = nullptr;
  return cudaSuccess;
}

// The checks and the launch that both entry points share.
static int layer_few(moe_plan* p, const void* x, const void* wr, const float* bias, LfMatrix wg, LfMatrix wu, LfMatrix wd, int group,
                     void* y, cudaStream_t st) {
  const moe_config_t& c = p->cfg;
  p->launches = 0;
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess) return MOE_ERR_CUDA;
  if (device != p->device) return MOE_ERR_ARG;
  if (c.T == 0) {  // no rows: no expert has any
    return cudaMemsetAsync(p->s.status, 0, 2 * sizeof(int), st) == cudaSuccess &&
                   cudaMemsetAsync(p->s.expert_count, 0, sizeof(int) * (size_t)c.E, st) == cudaSuccess
               ? MOE_OK
               : MOE_ERR_CUDA;
  }
  if (p->s.few_sync == nullptr) return MOE_ERR_WORKSPACE;
  // numbers of units and of rows are 32-bit
  const long long eb = c.dtype == MOE_DTYPE_BF16 ? 2 : 4, entries = min(2ll * p->route_E, (long long)c.T * p->route_K);
  if ((long long)c.T * c.H * eb >= 1ll << 31 || entries * kLfSlots * c.F * p->tp * eb >= 1ll << 31 || p->sm_count > 256) return MOE_ERR_UNSUPPORTED;
  LayerFewParams q = {};
  q.x = x;
  q.wr = wr;
  q.bias = bias;
  q.wg = wg;
  q.wu = wu;
  q.wd = wd;
  q.y = y;
  q.T = c.T;
  q.H = c.H;
  q.E = p->route_E;  // (an expert's TP shards lie next to one another in its matrices: here it is computed whole)
  q.K = p->route_K;
  q.F = c.F * p->tp;
  q.renorm = c.renormalize;
  q.tp = p->tp;
  // about a task per CTA, no slice under 256 columns; the scratch holds 256 sums per token
  q.slices = max(1, min(min(p->sm_count * kLfBatch, 256) / q.E, min(16, c.H / 256)));
  const int unit = 8;
  q.slice_cols = ((c.H + q.slices - 1) / q.slices + unit - 1) / unit * unit;
  q.slices = (c.H + q.slice_cols - 1) / q.slice_cols;
  q.split = split_outputs(p, group);
  q.partial = p->s.few_partial;
  q.logits = p->s.few_logits;
  q.inter = p->s.inter;
  q.sync = p->s.few_sync;
  q.topk_idx = p->s.topk_idx;
  q.topk_w = p->s.topk_w;
  q.expert_count = p->s.expert_count;
  q.status = p->s.status;
  q.wait_ns = c.wait_limit_ns ? c.wait_limit_ns : kDefaultWaitNs;
  const bool small = reading_us(p, group) < kSmallUs;
  cudaError_t e = few_start(p, st);
  if (e == cudaSuccess)
    e = group == 32    ? (small ? launch_cooperative<W4<32, true>>(p, q, st) : launch_cooperative<W4<32, false>>(p, q, st))
        : group == 64  ? (small ? launch_cooperative<W4<64, true>>(p, q, st) : launch_cooperative<W4<64, false>>(p, q, st))
        : group == 128 ? (small ? launch_cooperative<W4<128, true>>(p, q, st) : launch_cooperative<W4<128, false>>(p, q, st))
        : c.dtype != MOE_DTYPE_BF16 ? launch_cooperative<float>(p, q, st)
        : q.T > 4 && q.T * q.K >= 2 * q.E ? launch_cooperative<__nv_bfloat16, 2>(p, q, st) : launch_cooperative<__nv_bfloat16>(p, q, st);
  if (e != cudaSuccess) {
    cudaGetLastError();
    p->cuda_error = (int)e;
    p->cuda_error_step = 3;
    return MOE_ERR_CUDA;
  }
  p->launches = 1;
  return MOE_OK;
}

static int check_layer_few(const moe_plan* p, const void* x, const void* wr, const float* bias, const void* y) {
  if (!p || !wr) return MOE_ERR_ARG;
  if (p->cfg.T > 0 && (!x || !y)) return MOE_ERR_ARG;
  if (p->cfg.identity_experts) return MOE_ERR_ARG;
  if (p->cfg.T > MOE_FEW_MAX_TOKENS) return MOE_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(wr) | reinterpret_cast<uintptr_t>(y)) & 15) return MOE_ERR_ALIGN;
  if (reinterpret_cast<uintptr_t>(bias) & 3) return MOE_ERR_ALIGN;
  return MOE_OK;
}

}  // namespace moehub

using namespace moehub;

extern "C" {

int moe_layer_few(moe_plan_t* p, const void* d_x, const void* d_wr, const float* d_bias, const void* d_wg, const void* d_wu,
                  const void* d_wd, void* d_y, void* stream) {
  int rc = check_layer_few(p, d_x, d_wr, d_bias, d_y);
  if (rc != MOE_OK) return rc;
  if (!d_wg || !d_wu || !d_wd) return MOE_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(d_wg) | reinterpret_cast<uintptr_t>(d_wu) | reinterpret_cast<uintptr_t>(d_wd)) & 15) return MOE_ERR_ALIGN;
  return layer_few(p, d_x, d_wr, d_bias, {d_wg, nullptr}, {d_wu, nullptr}, {d_wd, nullptr}, 0, d_y, (cudaStream_t)stream);
}

int moe_layer_few_w4(moe_plan_t* p, const void* d_x, const void* d_wr, const float* d_bias, int32_t group, const moe_w4_t* wg,
                     const moe_w4_t* wu, const moe_w4_t* wd, void* d_y, void* stream) {
  int rc = check_layer_few(p, d_x, d_wr, d_bias, d_y);
  if (rc != MOE_OK) return rc;
  if (p->cfg.dtype != MOE_DTYPE_BF16) return MOE_ERR_UNSUPPORTED;
  const int F = p->cfg.F * p->tp;
  if ((rc = w4_check(wg, p->route_E, F, p->cfg.H, group)) != MOE_OK) return rc;
  if ((rc = w4_check(wu, p->route_E, F, p->cfg.H, group)) != MOE_OK) return rc;
  if ((rc = w4_check(wd, p->route_E, p->cfg.H, F, group)) != MOE_OK) return rc;
  auto matrix = [](const moe_w4_t* w) { return LfMatrix{w->codes, (const __nv_bfloat16*)w->scales}; };
  return layer_few(p, d_x, d_wr, d_bias, matrix(wg), matrix(wu), matrix(wd), group, d_y, (cudaStream_t)stream);
}

}  // extern "C"
