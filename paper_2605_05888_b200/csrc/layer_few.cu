// The whole MoE layer (paper Section II-A, steps 1-5) for a few tokens in one launch, on bf16, fp32 or 4-bit expert weights
// (moe_layer_few, moe_layer_few_w4 of include/moehub.h).
//
// As many CTAs as SMs, all resident (a cooperative launch), go through three parts with two grid-wide barriers between them:
//   router   every CTA forms the logits of a few experts, or of slices of them where there are few experts
//   gate/up  every CTA selects the picks for itself from the logits, and computes its share of the rows
//            S[u, t, f] = silu(x_t Wg[e_u, f]) * (x_t Wu[e_u, f]) of the used experts e_0 < e_1 < ...
//   down     every CTA computes its share of the outputs y[t, h] = sum_u w[u, t] sum_f S[u, t, f] Wd[e_u, h, f]: all the used
//            experts' columns of a row are in one CTA, so there is no separate combine step
// No row is copied, and no table is built that only a later launch would read.
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
  void* inter;             // [entries, 8, F]: the gate / up results of an entry's tokens
  unsigned* sync;          // two barriers: {arrived, generation} each
  int* topk_idx;           // the picks and rows per expert, as moe_layer leaves them (every TP shard listed)
  float* topk_w;
  int* expert_count;
  int* status;
  unsigned long long wait_ns;
};

// Every CTA of the grid arrives exactly once per launch and barrier, also one whose wait ran out before, so the counters are
// left as they were found whatever happens.  Everything written before is visible behind it (to loads that miss L1).
__device__ __forceinline__ void grid_barrier(const LayerFewParams& p, int which) {
  __syncthreads();
  if (threadIdx.x == 0) {
    unsigned* arrived = p.sync + 2 * which;
    int* generation = reinterpret_cast<int*>(p.sync + 2 * which + 1);
    const int before = ld_acquire(generation);
    __threadfence();
    if (atomicAdd(arrived, 1u) == gridDim.x - 1) {
      atomicExch(arrived, 0u);
      __threadfence();
      st_release(generation, before + 1);
    } else {
      const unsigned long long t0 = globaltimer();
      while (ld_acquire(generation) == before) {
        if (globaltimer() - t0 > p.wait_ns) {
          set_status(p.status, MOE_ERR_TIMEOUT, kWaitGrid);
          break;
        }
      }
    }
    __threadfence();
  }
  __syncthreads();
}

constexpr int kLfSlots = 8;      // tokens of an entry
constexpr int kLfEntries = 320;  // most entries: 256 experts, and 32 more eights of tokens among sixteen times 32 picks
struct LfShared {
  float w[kLfTokens * kLfPicks];                    // the picks' weights
  unsigned short used[kLfEntries];                  // an entry's expert, ascending
  unsigned char count[kLfEntries];
  unsigned char token[kLfEntries * kLfSlots];       // its tokens
  unsigned char pick[kLfEntries * kLfSlots];        // and which of a token's picks it is
  int warp_used[kMaxExperts / 32];
};
struct LfSelect {  // where the rows are streamed through later
  float red[kLfMaxWarps][kLfTokens];
  int idx[kLfTokens * kLfPicks];
  unsigned mask[kMaxExperts];
  int pos[kMaxExperts];  // a used expert's first entry
  float logits[kLfTokens * kMaxExperts];
};

// The logits (or a slice's part of them): a CTA per expert and slice, columns over its threads.
template <typename T>
__device__ __forceinline__ void lf_router(const LayerFewParams& p, LfSelect& s) {
  constexpr int N = Vec16<T>::N;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int task = blockIdx.x; task < p.E * p.slices; task += gridDim.x) {
    const int e = task / p.slices, slice = task % p.slices;
    const int c0 = slice * p.slice_cols, c1 = min(p.H, c0 + p.slice_cols);
    float acc[kLfTokens] = {};
    for (int c = c0 + (int)threadIdx.x * N; c < c1; c += blockDim.x * N) {
      float w[N];
      Vec16<T>::unpack(*reinterpret_cast<const uint4*>((const T*)p.wr + (size_t)e * p.H + c), w);
#pragma unroll
      for (int t = 0; t < kLfTokens; ++t) {
        if (t >= p.T) break;
        float v[N], part = 0.0f;
        Vec16<T>::unpack(*reinterpret_cast<const uint4*>((const T*)p.x + (size_t)t * p.H + c), v);
#pragma unroll
        for (int j = 0; j < N; ++j) part = __fmaf_rn(v[j], w[j], part);
        acc[t] += part;
      }
    }
#pragma unroll
    for (int t = 0; t < kLfTokens; ++t) {
      if (t >= p.T) break;
      const float sum = group_sum<32>(acc[t]);
      if (lane == 0) s.red[warp][t] = sum;
    }
    __syncthreads();
    if ((int)threadIdx.x < p.T) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < (int)blockDim.x / 32; ++i) sum += s.red[i][threadIdx.x];
      __stcg(p.logits + ((size_t)slice * p.T + threadIdx.x) * p.E + e, sum);
    }
    __syncthreads();
  }
}

// Every CTA selects for itself; returns the number of entries.
__device__ __forceinline__ int lf_select(const LayerFewParams& p, LfShared& s, LfSelect& q) {
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  for (int i = tid; i < p.T * p.E; i += blockDim.x) {
    float sum = 0.0f;
    for (int j = 0; j < p.slices; ++j) sum += __ldcg(p.logits + (size_t)j * p.T * p.E + i);
    q.logits[i] = p.bias != nullptr ? sum + p.bias[i % p.E] : sum;
  }
  if (tid < kMaxExperts) q.mask[tid] = 0;
  __syncthreads();
  if (p.E <= 64) select_topk<32, 2>(q.logits, p.E, p.T, 0, p.E, p.K, p.renorm, q.idx, s.w, nullptr, 1);
  else select_topk<32, 8>(q.logits, p.E, p.T, 0, p.E, p.K, p.renorm, q.idx, s.w, nullptr, 1);
  __syncthreads();
  for (int a = tid; a < p.T * p.K; a += blockDim.x) {
    atomicOr(&q.mask[q.idx[a]], 1u << (a / p.K));
    if (blockIdx.x == 0)
      for (int sh = 0; sh < p.tp; ++sh) {
        p.topk_idx[a * p.tp + sh] = q.idx[a] * p.tp + sh;
        p.topk_w[a * p.tp + sh] = s.w[a];
      }
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int e = tid; e < p.E * p.tp; e += blockDim.x) p.expert_count[e] = __popc(q.mask[e / p.tp]);
  // entries: one per used expert and eight tokens of it
  const int tokens = tid < kMaxExperts ? __popc(q.mask[tid]) : 0, entries = (tokens + kLfSlots - 1) / kLfSlots;
  int upto = entries;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, upto, off);
    if (lane >= off) upto += v;
  }
  if (lane == 31 && tid < kMaxExperts) s.warp_used[warp] = upto;
  __syncthreads();
  int pos = upto - entries, n = 0;
#pragma unroll
  for (int i = 0; i < kMaxExperts / 32; ++i) {
    if (i < warp) pos += s.warp_used[i];
    n += s.warp_used[i];
  }
  if (tid < kMaxExperts) q.pos[tid] = pos;
  for (int i = 0; i < entries; ++i) {
    s.used[pos + i] = (unsigned short)tid;
    s.count[pos + i] = (unsigned char)min(kLfSlots, tokens - i * kLfSlots);
  }
  __syncthreads();
  for (int a = tid; a < p.T * p.K; a += blockDim.x) {
    const int t = a / p.K, e = q.idx[a], slot = q.pos[e] * kLfSlots + __popc(q.mask[e] & ((1u << t) - 1u));
    s.token[slot] = (unsigned char)t;
    s.pick[slot] = (unsigned char)(a % p.K);
  }
  __syncthreads();
  return n;
}

__device__ __forceinline__ float lf_silu_mul(float g, float u) { return g / (1.0f + expf(-g)) * u; }

template <typename W>
__global__ void __launch_bounds__(RsSizes<W, 1>::THREADS, 1)
layer_few_kernel(const __grid_constant__ LayerFewParams p) {
  typedef typename RsFormat<W>::X X;
  typedef RsSizes<W, 1> Z;
  extern __shared__ __align__(128) unsigned char dynamic[];
  __shared__ LfShared s;
  static_assert(sizeof(LfSelect) <= Z::RING && Z::WARPS <= kLfMaxWarps && Z::THREADS >= kMaxExperts, "the selection's tables lie in the ring");
  LfSelect& q = *reinterpret_cast<LfSelect*>(dynamic);
  float* slots = reinterpret_cast<float*>(dynamic + Z::RING);
  const uint32_t ring = smem_u32(dynamic) + threadIdx.x / 32 * (Z::STAGES * Z::STAGE);
  const int lane = threadIdx.x % 32;
  if (blockIdx.x == 0 && threadIdx.x == 0) p.status[0] = p.status[1] = 0;
  lf_router<X>(p, q);
  grid_barrier(p, 0);
  const RsList list{s.used, s.count, s.token, lf_select(p, s, q)};

  // gate and up rows of the used experts
  const RsOperand gate_up{p.wg.w, p.wu.w, p.wg.scales, p.wu.scales, p.x, p.F, p.H, p.E};
  typedef RowStream<W, 1, kRsPairs> Up;
  Up up(gate_up, list, ring);
  auto finish_up = [&](int u, int row, int n0, int, const float*) {
#pragma unroll
    for (int j = 0; j < Z::REGS; ++j) {
      if (Up::kMma && j % 4 >= 2) continue;
      const float upper = Up::kMma ? up.acc[Up::kMma ? j + 2 : j] : __shfl_down_sync(0xffffffffu, up.acc[j], kRsRun);
      const int t = up.token(j), f = up.row_of(j);
      if (t < s.count[u] && f < n0 && (Up::kMma || lane < kRsRun))
        ((X*)p.inter)[((size_t)u * kLfSlots + t) * p.F + row + f] = from_float<X>(lf_silu_mul(up.acc[j], upper));
    }
  };
  up.run(nullptr, slots, [](int, int) { return 0.0f; }, finish_up);

  // the outputs; the first down rows are on their way while the other CTAs finish
  const RsOperand down_op{p.wd.w, p.wd.w, p.wd.scales, p.wd.scales, p.inter, p.H, p.F, p.E};
  typedef RowStream<W, 1, kRsSum> Down;
  Down down(down_op, list, ring);
  Down start = down;
  down.prefetch();
  __syncthreads();
  up.join(slots, finish_up);
  grid_barrier(p, 1);
  auto finish_down = [&](int, int row, int n0, int n1, const float* sums) {
    const int r = lane % kRsRun, first = lane < kRsRun ? row : row + n0;
    if (r < (lane < kRsRun ? n0 : n1))
      for (int t = 0; t < p.T; ++t) ((X*)p.y)[(size_t)t * p.H + first + r] = from_float<X>(sums[Down::sum_at(t, lane)]);
  };
  down.run(&start, slots, [&](int u, int slot) { return s.w[s.token[u * kLfSlots + slot] * p.K + s.pick[u * kLfSlots + slot]]; }, finish_down);
  __syncthreads();
  down.join(slots, finish_down);
}

template <typename W>
static cudaError_t launch_cooperative(const moe_plan* p, const LayerFewParams& q, cudaStream_t st) {
  static SmemAttrOnce once;
  auto kern = layer_few_kernel<W>;
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
// The checks and the launch that both entry points share.
static int layer_few(moe_plan* p, const void* x, const void* wr, const float* bias, LfMatrix wg, LfMatrix wu, LfMatrix wd, int group,
                     void* y, cudaStream_t st) {
  const moe_config_t& c = p->cfg;
  p->launches = 0;
  if (c.T == 0) return MOE_OK;
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess) return MOE_ERR_CUDA;
  if (device != p->device) return MOE_ERR_ARG;
  // the tokens' rows, and the gate / up results of at most two entries per expert, have 32-bit offsets
  const long long eb = c.dtype == MOE_DTYPE_BF16 ? 2 : 4, entries = min(2ll * p->route_E, (long long)c.T * p->route_K);
  if (c.T * c.H * eb >= 1ll << 32 || entries * kLfSlots * c.F * p->tp * eb >= 1ll << 32) return MOE_ERR_UNSUPPORTED;
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
  q.slices = max(1, min(min(p->sm_count, 256) / q.E, min(16, c.H / 256)));
  const int unit = 8;
  q.slice_cols = ((c.H + q.slices - 1) / q.slices + unit - 1) / unit * unit;
  q.slices = (c.H + q.slice_cols - 1) / q.slice_cols;
  q.logits = p->s.few_logits;
  q.inter = p->s.inter;
  q.sync = p->s.few_sync;
  q.topk_idx = p->s.topk_idx;
  q.topk_w = p->s.topk_w;
  q.expert_count = p->s.expert_count;
  q.status = p->s.status;
  q.wait_ns = c.wait_limit_ns ? c.wait_limit_ns : kDefaultWaitNs;
  cudaError_t e = group == 32 ? launch_cooperative<W4<32>>(p, q, st) : group == 64 ? launch_cooperative<W4<64>>(p, q, st) : group == 128 ? launch_cooperative<W4<128>>(p, q, st)
                  : c.dtype == MOE_DTYPE_BF16 ? launch_cooperative<__nv_bfloat16>(p, q, st) : launch_cooperative<float>(p, q, st);
  if (e != cudaSuccess) {
    cudaGetLastError();
    p->cuda_error = (int)e;
    p->cuda_error_step = 3;
    return MOE_ERR_CUDA;
  }
  p->launches = 1;
  return MOE_OK;
}

static int check_layer_few(const moe_plan* p, const void* x, const void* wr, const void* y) {
  if (!p || !wr) return MOE_ERR_ARG;
  if (p->cfg.T > 0 && (!x || !y)) return MOE_ERR_ARG;
  if (p->cfg.identity_experts) return MOE_ERR_ARG;
  if (p->cfg.T > MOE_FEW_MAX_TOKENS) return MOE_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(wr) | reinterpret_cast<uintptr_t>(y)) & 15) return MOE_ERR_ALIGN;
  return MOE_OK;
}

}  // namespace moehub

using namespace moehub;

extern "C" {

int moe_layer_few(moe_plan_t* p, const void* d_x, const void* d_wr, const float* d_bias, const void* d_wg, const void* d_wu,
                  const void* d_wd, void* d_y, void* stream) {
  int rc = check_layer_few(p, d_x, d_wr, d_y);
  if (rc != MOE_OK) return rc;
  if (!d_wg || !d_wu || !d_wd) return MOE_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(d_wg) | reinterpret_cast<uintptr_t>(d_wu) | reinterpret_cast<uintptr_t>(d_wd)) & 15) return MOE_ERR_ALIGN;
  return layer_few(p, d_x, d_wr, d_bias, {d_wg, nullptr}, {d_wu, nullptr}, {d_wd, nullptr}, 0, d_y, (cudaStream_t)stream);
}

int moe_layer_few_w4(moe_plan_t* p, const void* d_x, const void* d_wr, const float* d_bias, int32_t group, const moe_w4_t* wg,
                     const moe_w4_t* wu, const moe_w4_t* wd, void* d_y, void* stream) {
  int rc = check_layer_few(p, d_x, d_wr, d_y);
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
