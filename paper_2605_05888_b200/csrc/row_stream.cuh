// Products of matrix rows with a few operand rows ("tokens"), bound by reading the matrix once: what layer_few.cu and w4.cu share.
//
// A CTA has a range of matrix rows, cut into tiles of up to 32, and every tile into chunks of columns; its warps take equal,
// contiguous shares of all (tile, chunk) units, so that they have the same number of bytes to read whatever the sizes are.  Each warp
// copies its own units into its own ring of shared memory (16-byte asynchronous copies: bytes in flight without registers,
// no barrier between warps) and multiplies them by the tokens' columns: these come along in the stage, or (4 bits) straight into registers where they are needed.
// A tile that lies in one warp's share is finished from registers; of a tile that is cut, the warps after the first leave their
// sums in shared memory and the first adds them up, in order, so the sum does not depend on timing.
//
// The tensor cores' m16n8k16 (mma.sync) forms the products of bf16 and 4-bit rows: sixteen rows by eight tokens costs one
// instruction per 512 bytes of bf16 weights, so the multiplication is next to free, and the fragments come
// from shared memory without passing through tensor memory, which for tiles this thin would cost more than it gives (tcgen05's
// smallest tile has 64 rows: more than a CTA's share of the rows of small layers).  fp32 rows take plain FMAs, a lane per row.
#pragma once
#include "tc_common.cuh"
#include "w4_common.cuh"

namespace moehub {

constexpr int kRsTile = 32;   // rows of a tile: two runs of up to 16 consecutive rows
constexpr int kRsRun = 16;
constexpr int kRsRowBytes = 128;  // of a chunk

// 16 bytes into shared memory, past L1 (bytes 16), or zeros (bytes 0: nothing is read).  A row's next 128 bytes are asked into L2
// with these (Mixtral-like layer of 5 tokens: 378 us without, 339 with; DeepSeek-like of 16: 1357 and 1211).
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

// ---- the weights' formats ----------------------------------------------------------------------------------------------------
// 4 bits (float and __nv_bfloat16 name themselves).  SMALL: for little work, whose time the fetching of the code is a good part of (every SM
// fetches it, also from HBM): half a chunk's code is not unrolled twice, and runs of at most eight rows have a form of their own.  For much
// work that form costs more than it saves, since it is rarely taken.
template <int GROUP, bool SMALL> struct W4 {};
template <typename W> struct RsFormat;
template <> struct RsFormat<__nv_bfloat16> {
  typedef __nv_bfloat16 X;                       // the tokens' type
  static constexpr int COLS = 64;                // columns of a chunk: 128 bytes of a row
  static constexpr int GROUP = 1, GROUPS = 0;    // (4 bits) columns of a group, groups of a chunk
  static constexpr int WARPS = 8;
};
template <> struct RsFormat<float> {
  typedef float X;
  static constexpr int COLS = 32, GROUP = 1, GROUPS = 0, WARPS = 8;
};
template <int G, bool S> struct RsFormat<W4<G, S>> {
  typedef __nv_bfloat16 X;
  static constexpr bool SMALL = S;
  static constexpr int COLS = 256, GROUP = G, GROUPS = COLS / G;
  // Of about 20 instructions per word of eight codes 12 unpack and multiply it (3 shifts, 4 masks, 4 subtractions, an MMA).  No unit is full (55 % of the issue
  // slots, 55 % of the ALU, HBM at 48 %): latencies count, so the more warps the better, as long as their registers suffice (at 16 the layers' code for
  // groups of 64 and 32 spills 44 and 16 bytes, that for 128 nothing).  Mixtral-like layer of 7 tokens, us, 8 / 12 / 16 warps: 234 / 186 / 170.  An earlier form of the loop
  // took 181: without unpacking 167, without the tokens' loads 166, without the scales 178, without all three 129 (116 for the bytes).
  static constexpr int WARPS = 16;
};
template <typename W, int NT> struct RsSizes {   // NT: token slots, in eights
  typedef RsFormat<W> F;
  static constexpr int WARPS = NT == 1 ? F::WARPS : 8, THREADS = 32 * WARPS;
  static constexpr int A = kRsTile * kRsRowBytes;
  static constexpr int X = F::GROUPS == 0 ? 8 * NT * kRsRowBytes : 0;
  static constexpr int SCALES = F::GROUPS * 2 * 9 * 4;  // per group two runs of nine words (16 scales from an odd one on)
  static constexpr int STAGE = (A + X + SCALES + 127) / 128 * 128;
  static constexpr int REGS = 8 * NT;            // sums per lane
  static constexpr int SLOT = 16 * kRsTile;      // floats of a warp's slot: its sums of a tile, or (kRsSum) 16 tokens' sums of its rows
  static constexpr int SLOTS = WARPS * SLOT * 4;
  static constexpr int ROOM = 218 * 1024 - SLOTS;  // (9 KB are left for the kernels' own tables)
  static constexpr int STAGES = ROOM / WARPS / STAGE < 6 ? ROOM / WARPS / STAGE : 6;
  static constexpr int WARP_RING = ROOM / WARPS / 128 * 128;  // (of either NT's streams in one kernel)
  static constexpr int RING = WARPS * WARP_RING;
  static constexpr int BYTES = RING + SLOTS;     // dynamic shared memory
  static_assert(STAGES >= 2 && REGS * 32 <= SLOT && STAGES * STAGE >= SLOT * 4, "a stage to fill beside one to read; a tile's sums fit a slot, a slot the ring");
};

// A product's matrices and tokens.
struct RsOperand {
  const void* w0;               // rows of run 0: [matrices, N, C]
  const void* w1;               // rows of run 1 (gate / up: the other matrix's; else w0)
  const __nv_bfloat16* s0;      // 4 bits: scales [matrices, C / group, N]
  const __nv_bfloat16* s1;
  const void* x;                // token rows [.., C]
  long long x_rest;             // kRsSum on tensor cores: elements from a token's row to the row of what rounding it to bf16 left
  int N, C, matrices;           // matrices: all there are
  int split;                    // kRsSum: 1: all CTAs' warps share all rows' units, so that a tile's sums may lie in several CTAs; 0: a CTA has rows of its own
};

// What is to be multiplied: entries, each a matrix and the few tokens that it is for (a matrix with more tokens has several
// entries, which share its reading in L2).  In shared memory.
// An entry has up to 8 * NT tokens, a slot each; in kRsSum on tensor cores half as many.  The tokens there are results of another product, and
// come as two bf16 numbers each, what a value rounds to and what that left, in slots s and 4 * NT + s: so the rounding does not show in
// the outputs (with one number each they were 0.0024 from the sums in 64 bits, with two 0.0017, which is their own rounding), and
// costs nothing while slots are free.
struct RsList {
  const unsigned short* used;   // matrix of an entry
  const unsigned char* count;   // its tokens
  const unsigned char* token;   // [8 * NT] per entry: the rows of x (not kRsSum)
  const unsigned short* row;    // kRsSum: the first token's row of x, the others follow
  int n;
};

// n things in `parts` shares that differ by one at most: where share i begins and how many it has.  (32 bits and one division: the
// kernels' latencies are made of such.)
struct RsShare {
  int begin, count;
  __device__ __forceinline__ RsShare(unsigned n, unsigned parts, unsigned i) {
    const unsigned each = n / parts, more = n - each * parts;
    begin = (int)(each * i + min(i, more));
    count = (int)(each + (i < more ? 1 : 0));
  }
  // The share that thing `at` is in.
  __device__ __forceinline__ static int of(unsigned n, unsigned parts, unsigned at) {
    const unsigned each = n / parts, more = n - each * parts, line = more * (each + 1);
    return (int)(at < line ? at / (each + 1) : more + (at - line) / each);
  }
};

// The rows of one CTA (or of all, `groups` 1): its share of `used` entries' rows laid end to end (fewer than 2^31).  RT: rows of a tile.
struct RsRange {
  int end, N, RT, first_u, first_row, first_len, first_tiles, full_tiles, tiles;
  __device__ __forceinline__ RsRange(int used, int N_, int RT_, unsigned group, unsigned groups) : N(N_), RT(RT_) {
    const RsShare mine(group < groups ? (unsigned)(used * N) : 0u, groups, group);
    tiles = 0;
    if (mine.count == 0) return;
    end = mine.begin + mine.count;
    first_u = (unsigned)mine.begin / (unsigned)N;
    first_row = mine.begin - first_u * N;
    first_len = min(mine.count, N - first_row);
    first_tiles = (first_len + RT - 1) / RT;
    full_tiles = (N + RT - 1) / RT;
    tiles = first_tiles;
    const int rest = mine.count - first_len;
    if (rest > 0) {
      const int whole = (unsigned)rest / (unsigned)N;
      tiles += whole * full_tiles + (rest - whole * N + RT - 1) / RT;
    }
  }
  // entry, first row and number of rows of tile i
  __device__ __forceinline__ void tile(int i, int& u, int& row, int& n) const {
    int start = first_row, len = first_len, count = first_tiles, k = i;
    u = first_u;
    if (i >= first_tiles) {
      const int j = i - first_tiles, skip = (unsigned)j / (unsigned)full_tiles;
      u += 1 + skip;
      k = j - skip * full_tiles;
      start = 0;
      len = min(N, end - u * N);
      count = (len + RT - 1) / RT;
    }
    const RsShare rows(len, count, k);
    row = start + rows.begin;
    n = rows.count;
  }
};

enum RsKind {
  kRsPairs,   // tiles of up to 16 pairs: row f of w0 and row f of w1, of one entry each
  kRsRows,    // tiles of up to 32 rows of one entry each
  kRsSum,     // tiles of up to 32 rows, the same rows of every entry one after the other, weighted and added per token
};

// A warp's way through its units.
template <typename W, int NT, int KIND>
struct RowStream {
  typedef RsFormat<W> F;
  typedef RsSizes<W, NT> Z;
  typedef typename F::X X;
  static constexpr int REGS = Z::REGS, WARPS = Z::WARPS, SLOTS = 8 * NT;
  static constexpr bool kMma = sizeof(X) == 2;
  static constexpr bool k4Bit = F::GROUPS > 0;
  static constexpr int RPI = 4;                   // rows of a copy instruction: eight lanes each
  static constexpr int HALF = 128;                // (4 bits) columns whose tokens are in registers: half a chunk

  const RsOperand& op;
  const RsList& list;
  RsRange range;
  int chunks, per_tile;      // chunks of a matrix row, of a tile
  int total, left;           // units of the share; how many are still to be copied
  // where the copies are
  int tile_i, chunk, u, row, n0, n1;  // chunk: of the matrix
  const char *pa0, *pa1;     // the lane's first bytes of the unit (4 bits: pa1 comes from pa0, for the registers)
  const char* ps;            // (4 bits, N even) the lane's scale word of the unit's first group
  bool has_scale;
  const char* px[2 * NT];    // (not 4 bits) the lane's bytes of tokens lane / 8, 4 + lane / 8, ..
  uint32_t ring;             // shared address of the warp's ring
  int lane;

  __device__ __forceinline__ RowStream(const RsOperand& op_, const RsList& list_, uint32_t ring_)
      : op(op_), list(list_), range(KIND == kRsSum ? 1 : list_.n, op_.N, KIND == kRsPairs ? kRsRun : kRsTile, op_.split ? 0 : blockIdx.x, op_.split ? 1 : gridDim.x), ring(ring_) {
    lane = threadIdx.x % 32;
    chunks = (op.C + F::COLS - 1) / F::COLS;
    per_tile = KIND == kRsSum ? chunks * list.n : chunks;
    const RsShare mine = share(threadIdx.x / 32);
    total = left = mine.count;
    if (left > 0) {
      tile_i = (unsigned)mine.begin / (unsigned)per_tile;
      const int c = mine.begin - tile_i * per_tile;
      set_tile(tile_i, u, row, n0, n1);
      if (KIND == kRsSum) u = (unsigned)c / (unsigned)chunks;
      chunk = KIND == kRsSum ? c - u * chunks : c;
      set_pointers();
    }
  }

  __device__ __forceinline__ RsShare share(int warp) const {
    const int first = KIND == kRsSum && op.split ? blockIdx.x * WARPS : 0;
    return RsShare(range.tiles * per_tile, shares(), first + warp);
  }
  __device__ __forceinline__ unsigned shares() const { return KIND == kRsSum && op.split ? WARPS * gridDim.x : WARPS; }
  // (split) Which CTA has a unit.
  __device__ __forceinline__ int cta_of(int unit) const { return RsShare::of(range.tiles * per_tile, shares(), unit) / WARPS; }

  __device__ __forceinline__ void set_tile(int i, int& tu, int& trow, int& tn0, int& tn1) const {
    int n;
    range.tile(i, tu, trow, n);
    if (KIND == kRsPairs) tn0 = tn1 = n;
    else { tn0 = (n + 1) / 2; tn1 = n - tn0; }
  }
  // The second run's first row.
  __device__ __forceinline__ static int row1(int r, int m0) { return KIND == kRsPairs ? r : r + m0; }

  __device__ __forceinline__ long long row_bytes() const { return k4Bit ? op.C / 2 : (long long)op.C * (int)sizeof(X); }
  __device__ __forceinline__ void set_pointers() {
    const long long e = list.used[u], ld = row_bytes();
    const long long at = (long long)(lane / 8) * ld + (long long)chunk * kRsRowBytes + lane % 8 * 16;
    pa0 = (const char*)op.w0 + (e * op.N + row) * ld + at;
    if constexpr (!k4Bit) pa1 = (const char*)op.w1 + (e * op.N + row1(row, n0)) * ld + at;
    if constexpr (!k4Bit)
#pragma unroll
      for (int i = 0; i < 2 * NT; ++i)
        px[i] = (const char*)((const X*)op.x + x_row(u, i * 4 + lane / 8)) + (long long)chunk * kRsRowBytes + lane % 8 * 16;
    if constexpr (k4Bit) {
      const int r = lane < 16 ? row : row1(row, n0);
      const long long first = (e * (op.C / F::GROUP) + (long long)chunk * F::GROUPS) * op.N + r;
      ps = (const char*)((lane < 16 ? op.s0 : op.s1) + (first & ~1ll) + 2 * (lane % 16));
      has_scale = lane % 16 < 9 && 2 * (lane % 16) < (lane < 16 ? n0 : n1) + (r & 1);
    }
  }
  static constexpr bool kTwo = KIND == kRsSum && kMma;  // tokens as two numbers
  // Where the row of x for an entry's slot begins (for one without a token: the first's), in elements.
  __device__ __forceinline__ long long x_row(int mu, int slot) const {
    const int s = kTwo ? slot % (SLOTS / 2) : slot, t = s < list.count[mu] ? s : 0;
    return (long long)(KIND == kRsSum ? (int)list.row[mu] + t : (int)list.token[mu * SLOTS + t]) * op.C + (kTwo && slot >= SLOTS / 2 ? op.x_rest : 0);
  }

  __device__ __forceinline__ void advance() {
    --left;
    pa0 += kRsRowBytes;
    if constexpr (!k4Bit) pa1 += kRsRowBytes;
    if constexpr (!k4Bit)
#pragma unroll
      for (int i = 0; i < 2 * NT; ++i) px[i] += kRsRowBytes;
    if constexpr (k4Bit) ps += 2ll * F::GROUPS * op.N;
    if (++chunk == chunks && left > 0) {
      chunk = 0;
      if (KIND == kRsSum && u + 1 < list.n) {
        ++u;
      } else {
        set_tile(++tile_i, u, row, n0, n1);
        if (KIND == kRsSum) u = 0;
      }
      set_pointers();
    }
  }

  __device__ __forceinline__ const char* second() const {
    if constexpr (!k4Bit) return pa1;
    return KIND == kRsPairs ? pa0 + ((const char*)op.w1 - (const char*)op.w0) : pa0 + n0 * row_bytes();
  }

  // The weights (and scales) of the current unit into a stage; zeros beyond the row.
  __device__ __forceinline__ void copy_weights(uint32_t dst) const {
    const long long step = RPI * row_bytes();
    const int bytes = chunk * kRsRowBytes + lane % 8 * 16 < (int)row_bytes() ? 16 : 0;
    const char *a0 = pa0, *a1 = second();
    const int limit0 = n0 - lane / 8, limit1 = n1 - lane / 8;
#pragma unroll
    for (int i = 0; i < kRsRun / RPI; ++i) {
      const int r = i * RPI + lane / 8;
      const uint32_t at = dst + place(r, lane % 8);
      if (i * RPI < limit0) copy16(at, a0, bytes);
      if (i * RPI < limit1) copy16(at + kRsRun * kRsRowBytes, a1, bytes);
      a0 += step;
      a1 += step;
    }
    if constexpr (k4Bit) copy_scales(dst + Z::A);
  }
  // Where 16-byte unit c of a row is, so that eight rows' same unit lie in different banks.
  __device__ __forceinline__ static int place(int r, int c) { return r * kRsRowBytes + ((c ^ (r & 7)) * 16); }

  // (4 bits) Whether N is odd: only in products by themselves.  (A layer's N are other matrices' C, multiples of the group; without the code for
  // it a layer of 7 Mixtral-like tokens takes 172 us, with it 179.)
  __device__ __forceinline__ bool odd() const { return KIND == kRsRows && (op.N & 1); }

  // Scale words: [group of the chunk][run][9], 16 rows from an even element on; half a warp per run.
  __device__ __forceinline__ void copy_scales(uint32_t dst) const {
    const int G = op.C / F::GROUP, i = lane % 16;
    dst += lane / 16 * 36 + i * 4;
    if (!odd()) {  // every group's scales begin like the first's
      const char* s = ps;
#pragma unroll
      for (int q = 0; q < F::GROUPS; ++q) {
        if (has_scale) copy4(dst + q * 72, s, chunk * F::GROUPS + q < G ? 4 : 0);
        s += 2ll * op.N;
      }
      return;
    }
    const int n = lane < 16 ? n0 : n1;
    const long long all = (long long)op.matrices * G * op.N;
    const __nv_bfloat16* s = lane < 16 ? op.s0 : op.s1;
    long long first = ((long long)list.used[u] * G + chunk * F::GROUPS) * op.N + (lane < 16 ? row : row1(row, n0));
#pragma unroll
    for (int q = 0; q < F::GROUPS; ++q) {
      const long long at = (first & ~1ll) + 2 * i;
      const bool some = chunk * F::GROUPS + q < G && 2 * i < n + (int)(first & 1);
      if (i < 9) copy4(dst + q * 72, some ? s + at : s, some ? (at + 1 < all ? 4 : 2) : 0);
      first += op.N;
    }
  }

  // The tokens' columns of the current unit (4 bits: see fetch_tokens).
  __device__ __forceinline__ void copy_tokens(uint32_t dst) const {
    if constexpr (!k4Bit) {
      const int bytes = chunk * kRsRowBytes + lane % 8 * 16 < (int)row_bytes() ? 16 : 0, limit = (int)list.count[u] - lane / 8;
#pragma unroll
      for (int i = 0; i < 2 * NT; ++i)
        if ((kTwo ? i * 4 % (SLOTS / 2) : i * 4) < limit) copy16(dst + Z::A + place(i * 4 + lane / 8, lane % 8), px[i], bytes);
    }
  }
  // 4 bits: the lane's columns 8 * (lane % 4) and on of each 32, of half a chunk, of token lane / 4.
  __device__ __forceinline__ void fetch_tokens(int half, uint4 (&b)[NT][4]) const {
    const int c = m_chunk * F::COLS + half * HALF;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint4* from = reinterpret_cast<const uint4*>(m_x[t] + c);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        b[t][k] = make_uint4(0, 0, 0, 0);
        if (c + 32 * k < op.C) b[t][k] = KIND == kRsSum ? __ldcg(from + 4 * k) : __ldg(from + 4 * k);  // (kRsSum: written by this launch)
      }
    }
  }

  // A stage's products added to acc.  MT (tensor cores): 1 where the runs have at most 8 rows, else 2.  fp32: a lane per row, also where the
  // runs have few rows.  (Slots without a token hold anything: their
  // sums are not read.)
  template <int MT>
  __device__ __forceinline__ void multiply(uint32_t a, int tokens) {
    if constexpr (!kMma) {
      float w[32];
#pragma unroll
      for (int c = 0; c < 8; ++c) Vec16<float>::unpack(lds128(a + place(lane, c)), w + 4 * c);
#pragma unroll
      for (int t = 0; t < SLOTS; ++t) {
        if (t >= tokens) break;
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          float v[4];
          Vec16<float>::unpack(lds128(a + Z::A + place(t, c)), v);
          s0 = __fmaf_rn(w[4 * c], v[0], s0);
          s1 = __fmaf_rn(w[4 * c + 1], v[1], s1);
          s0 = __fmaf_rn(w[4 * c + 2], v[2], s0);
          s1 = __fmaf_rn(w[4 * c + 3], v[3], s1);
        }
        acc[t] += s0 + s1;
      }
    } else {
      uint32_t b[NT][4][2];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t r[4];
          ldsm4(a + Z::A + 8 * t * kRsRowBytes + place(lane % 8, 4 * q + lane / 8), r);
          b[t][2 * q][0] = r[0]; b[t][2 * q][1] = r[1]; b[t][2 * q + 1][0] = r[2]; b[t][2 * q + 1][1] = r[3];
        }
      // The chunk's sums, added to the others in fp32: an MMA cuts off what its sum cannot hold, towards zero, so that a chain over a whole row
      // loses a part of itself with every instruction (65536 cancelling terms: 1109 times 2^-24 of the largest partial sum by a chain, 3 so;
      // 0.1 to 0.7 % of a layer's time).
      float part[MT][NT][4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          uint32_t w[4];
          ldsm4(a + (lane / 8 % 2 * kRsRun + 8 * m) * kRsRowBytes + place(lane % 8, 2 * k + lane / 16), w);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            if (k == 0) mma16816_first(part[m][t], w[0], w[1], w[2], w[3], b[t][k][0], b[t][k][1]);
            else mma16816(part[m][t], w[0], w[1], w[2], w[3], b[t][k][0], b[t][k][1]);
          }
        }
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) sums(m, t)[i] += part[m][t][i];
    }
  }
  __device__ __forceinline__ float (&sums(int m, int t))[4] { return reinterpret_cast<float(&)[4]>(acc[(m * NT + t) * 4]); }

  // Half a stage's products on 4-bit rows.  at: the lane's first row address (ldmatrix); s0, s1: of the runs' scales of the half's
  // groups 0, 2, ..; f0, f1: 2 or 0 bytes, to be flipped for groups 1, 3, ..
  template <int MT>
  __device__ __forceinline__ void multiply4(uint32_t at, const uint4 (&b)[NT][4], uint32_t s0, uint32_t s1, uint32_t f0, uint32_t f1) {
    constexpr int per_group = F::GROUP / 32;  // 32-column units
    float part[MT][NT][4];
    uint32_t w[MT][2][4];
    float e[MT][2][4 / per_group];  // the scales, ahead of their use
#pragma unroll
    for (int q = 0; q < 4 / per_group; ++q)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        e[m][0][q] = scale(s0 + q * 72 + 16 * m + (q % 2 ? f0 : 0));
        e[m][1][q] = scale(s1 + q * 72 + 16 * m + (q % 2 ? f1 : 0));
      }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int m = 0; m < MT; ++m) ldsm4((k == 0 ? at : at ^ 32u) + 8 * m * kRsRowBytes, w[m][k]);  // (stages are 128-byte aligned)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        uint32_t d0[4], d1[4];
        dequantise(w[m][k / 2][k % 2 * 2], d0);
        dequantise(w[m][k / 2][k % 2 * 2 + 1], d1);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (k % per_group == 0) mma16816_first(part[m][t], d0[0], d1[0], d0[1], d1[1], b[t][k].x, b[t][k].y);
          else mma16816(part[m][t], d0[0], d1[0], d0[1], d1[1], b[t][k].x, b[t][k].y);
          mma16816(part[m][t], d0[2], d1[2], d0[3], d1[3], b[t][k].z, b[t][k].w);
        }
      }
      if ((k + 1) % per_group == 0) {   // the group's sums, scaled once
        const int q = k / per_group;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const float e0 = e[m][0][q], e1 = e[m][1][q];
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            float(&s)[4] = sums(m, t);
            s[0] = __fmaf_rn(e0, part[m][t][0], s[0]);
            s[1] = __fmaf_rn(e0, part[m][t][1], s[1]);
            s[2] = __fmaf_rn(e1, part[m][t][2], s[2]);
            s[3] = __fmaf_rn(e1, part[m][t][3], s[3]);
          }
        }
      }
    }
  }
  __device__ __forceinline__ void multiply_codes(uint32_t a) {
    const uint32_t at = a + (lane / 8 % 2 * kRsRun) * kRsRowBytes + place(lane % 8, lane / 16), sc = a + Z::A + lane / 4 * 2;
    // a run's scale of group g is number (matrix's + g) * N + row: whether it lies in the second half of its first word
    uint32_t o0 = m_row & 1 ? 2u : 0u, o1 = row1(m_row, m_n0) & 1 ? 2u : 0u, flip = 0;
    if (odd()) {
      flip = 2;
      if ((m_base + m_chunk * F::GROUPS) & 1) { o0 ^= 2u; o1 ^= 2u; }
    }
#pragma unroll (F::SMALL ? 1 : 2)
    for (int half = 0; half < 2; ++half) {
      if (m_chunk * F::COLS + half * HALF >= op.C) break;
      uint4 b[NT][4];
      fetch_tokens(half, b);
      if (half == 0) {
        copies_wait<Z::STAGES - 1>();
        __syncwarp();
      } else if (F::GROUPS == 2) {  // (an odd number of groups on)
        o0 ^= flip;
        o1 ^= flip;
      }
      const uint32_t s0 = sc + half * (F::GROUPS * 36) + o0, s1 = sc + half * (F::GROUPS * 36) + 36 + o1;
      const uint32_t f0 = flip == 0 ? 0 : o0 ? (uint32_t)-2 : 2, f1 = flip == 0 ? 0 : o1 ? (uint32_t)-2 : 2;
      if (F::SMALL && m_n0 <= 8) multiply4<1>(at ^ (half * 64), b, s0, s1, f0, f1);
      else multiply4<2>(at ^ (half * 64), b, s0, s1, f0, f1);
    }
  }
  // Eight codes as exact bf16 integers code - 8, in pairs of neighbouring columns: 128 + code has the code in its last bits.
  __device__ __forceinline__ static void dequantise(uint32_t word, uint32_t (&d)[4]) {
    const __nv_bfloat162 bias = __halves2bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308));  // 136
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t v;
      asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(v) : "r"(word >> (4 * i)));
      const __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&v), bias);
      d[i] = *reinterpret_cast<const uint32_t*>(&r);
    }
  }
  __device__ __forceinline__ static float scale(uint32_t at) {
    unsigned short v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
    return __uint_as_float((uint32_t)v << 16);
  }

  // ---- the warp's loop: prefetch() [the weights alone, before the tokens exist], run(), then a barrier of the CTA, then join() ----

  // Where the products are; what run() leaves of a tile that goes on in the next warps' shares.
  int m_tile, m_u, m_chunk, m_row, m_n0, m_n1, m_base, m_tokens;
  const X* m_x[NT];  // (4 bits) the lane's first column of its tokens
  bool pending;
  float acc[REGS];

  __device__ __forceinline__ void prefetch() {
    __syncwarp();
#pragma unroll 1
    for (int i = 0; i < Z::STAGES - 1; ++i)
      if (left > 0) {
        copy_weights(ring + i * Z::STAGE);
        advance();
      }
    copies_commit();
  }

  __device__ __forceinline__ void set_matrix() {
    m_tokens = list.count[m_u];
    if constexpr (k4Bit)
#pragma unroll
      for (int t = 0; t < NT; ++t) m_x[t] = (const X*)op.x + x_row(m_u, 8 * t + lane / 4) + lane % 4 * 8;
    if constexpr (k4Bit) m_base = list.used[m_u] * (op.C / F::GROUP);
  }
  // Sums of tokens' first numbers and of what rounding left.  A weight that is an infinity makes the first an infinity, or a NaN where the
  // token has a zero; the second, of numbers of any sign and zeros, would make a NaN of the infinity.
  __device__ __forceinline__ static float with_rest(float near, float rest) { return fabsf(near) < INFINITY ? near + rest : near; }
  // kRsSum: where a warp adds up its rows' results per token.  (The rows are swizzled so that the lanes of a fragment, which
  // hold eight rows of four tokens, hit different banks.)
  __device__ __forceinline__ static int sum_at(int t, int r) { return t * kRsTile + (r ^ ((t & 3) << 3)); }

  // start: a copy of this stream as it was before prefetch(), or nullptr without one.  weight(u, t, token&): of
  // an entry's token t, and which it is among the outputs (kRsSum).  finish(u, row, n0, n1, sums): a whole tile, whose sums are in acc or (kRsSum) in shared memory at sum_at().
  // slots: shared memory, Z::SLOTS bytes.
  template <typename Weight, typename Finish>
  __device__ __forceinline__ void run(RowStream* start, float* slots, Weight weight, Finish finish) {
    const RowStream& at = start != nullptr ? *start : *this;
    m_tile = at.tile_i; m_u = at.u; m_chunk = at.chunk; m_row = at.row; m_n0 = at.n0; m_n1 = at.n1;
    pending = false;
    if (total <= 0) {
      copies_wait<0>();
      return;
    }
    set_matrix();
    float* slot = slots + threadIdx.x / 32 * Z::SLOT;
    bool cut = KIND == kRsSum ? m_u != 0 || m_chunk != 0 : m_chunk != 0;  // the tile begins in an earlier warp's share
    float held[Z::SLOT / 32];
    bool hold = false;
#pragma unroll 1
    for (int i = 0; i < Z::STAGES - 1; ++i) {
      if (i < total) {
        if (start != nullptr) {
          start->copy_tokens(ring + i * Z::STAGE);
          start->advance();
        } else {
          copy_weights(ring + i * Z::STAGE);
          copy_tokens(ring + i * Z::STAGE);
          advance();
        }
      }
      copies_commit();
    }
#pragma unroll
    for (int j = 0; j < REGS; ++j) acc[j] = 0.0f;
    if (KIND == kRsSum)
      for (int j = lane; j < Z::SLOT; j += 32) slot[j] = 0.0f;
    uint32_t stage = ring, next = ring + (Z::STAGES - 1) * Z::STAGE;
#pragma unroll 1
    for (int i = 0; i < total; ++i) {
      __syncwarp();
      if (left > 0) {
        copy_weights(next);
        copy_tokens(next);
        advance();
      }
      copies_commit();
      if constexpr (k4Bit) {
        multiply_codes(stage);
      } else {
        copies_wait<Z::STAGES - 1>();
        __syncwarp();
        if constexpr (kMma) {
          if (m_n0 > 8) multiply<2>(stage, m_tokens);
          else multiply<1>(stage, m_tokens);
        } else {
          multiply<1>(stage, m_tokens);
        }
      }
      next = stage;
      stage = stage + Z::STAGE == ring + Z::STAGES * Z::STAGE ? ring : stage + Z::STAGE;
      ++m_chunk;
      const bool last = i + 1 == total;
      if (m_chunk < chunks && !last) continue;
      // the end of a matrix's columns, or of the share
      if (KIND == kRsSum) {
#pragma unroll
        for (int j = 0; j < REGS; ++j) {
          const int t = token(j);
          if (kTwo && NT == 1) acc[j] = with_rest(acc[j], __shfl_xor_sync(0xffffffffu, acc[j], 2));  // slots s and 4 + s
          if (kTwo && NT == 2 && j / 4 % NT == 0) acc[j] = with_rest(acc[j], acc[j + 4]);            // s and 8 + s
          if (t < m_tokens) {
            int to_token;
            const float w = weight(m_u, t, to_token);
            float* to = slot + sum_at(to_token, run_of(j) * kRsRun + row_of(j));
            *to = __fmaf_rn(w, acc[j], *to);
          }
          if (!(kTwo && NT == 2)) acc[j] = 0.0f;
        }
        if (kTwo && NT == 2)
#pragma unroll
          for (int j = 0; j < REGS; ++j) acc[j] = 0.0f;
        __syncwarp();
        if (m_chunk == chunks && m_u + 1 < list.n) {
          ++m_u;
          m_chunk = 0;
          set_matrix();
          if (!last) continue;
        }
      }
      if (cut) {
        if (KIND == kRsSum) {
#pragma unroll
          for (int j = 0; j < Z::SLOT / 32; ++j) held[j] = slot[j * 32 + lane];
          hold = true;
        } else {
#pragma unroll
          for (int j = 0; j < REGS; ++j) slot[j * 32 + lane] = acc[j];
        }
      } else if (m_chunk == chunks) {  // (kRsSum: of the last entry)
        finish(m_u, m_row, m_n0, m_n1, slot);
      } else {
        pending = true;
      }
      if (!last) {  // (the tile was whole, or its end)
        cut = false;
        m_chunk = 0;
        set_tile(++m_tile, m_u, m_row, m_n0, m_n1);
        if (KIND == kRsSum) {
          m_u = 0;
          __syncwarp();
          for (int j = lane; j < Z::SLOT; j += 32) slot[j] = 0.0f;
          __syncwarp();
        }
#pragma unroll
        for (int j = 0; j < REGS; ++j) acc[j] = 0.0f;
        set_matrix();
      }
    }
    copies_wait<0>();
    if (KIND == kRsSum && hold) {  // the ring is free now
      __syncwarp();
      float* area = held_area(threadIdx.x / 32);
#pragma unroll
      for (int j = 0; j < Z::SLOT / 32; ++j) area[j * 32 + lane] = held[j];
    }
  }

  // Behind the barrier: what the warps hold of cut tiles is added up in the warps' order and finished.
  // kRsPairs, kRsRows: by the warp that the tile begins in, by finish as above.
  template <typename Finish>
  __device__ __forceinline__ void join(float* slots, Finish finish) {
    if (!pending) return;
    const int tile_end = (m_tile + 1) * per_tile;
    for (int w = threadIdx.x / 32 + 1; w < WARPS; ++w) {
      const RsShare s = share(w);
      if (s.begin >= tile_end) break;
      if (s.count == 0) continue;
#pragma unroll
      for (int j = 0; j < REGS; ++j) acc[j] += slots[w * Z::SLOT + j * 32 + lane];
    }
    finish(m_u, m_row, m_n0, m_n1, slots);
  }
  // kRsSum: by all threads, a value each; store(row of y, token, value, part).  (split) part: the CTA's number among those that have some of
  // the tile (0 where finish gets a tile: it is whole); combine() adds them up.
  template <typename Store>
  __device__ __forceinline__ void join_sums(const float* slots, int tokens, Store store) {
    int i = 0, end = range.tiles;
    if (op.split) {
      const RsShare first = share(0), last = share(WARPS - 1);
      if (first.count == 0) return;
      i = (unsigned)first.begin / (unsigned)per_tile;
      end = (unsigned)(last.begin + last.count - 1) / (unsigned)per_tile + 1;
    }
    for (; i < end; ++i) {
      const int lo = i * per_tile, hi = lo + per_tile, part = op.split ? blockIdx.x - cta_of(lo) : 0;
      int tu, row0, m0, m1;
      set_tile(i, tu, row0, m0, m1);
      for (int at = threadIdx.x; at < tokens * kRsTile; at += Z::THREADS) {
        const int t = at / kRsTile, r = at % kRsTile;
        float v = 0.0f;
        bool whole = false;
#pragma unroll 4
        for (int w = 0; w < WARPS; ++w) {
          const RsShare s = share(w);
          const int s_end = s.begin + s.count;
          if (s.count == 0 || s_end <= lo || s.begin >= hi) continue;
          whole = s.begin <= lo && s_end >= hi;  // (finished by its warp)
          if (!whole) v += (s.begin > lo ? held_area(w) : slots + w * Z::SLOT)[sum_at(t, r)];
        }
        const int k = r % kRsRun;
        if (!whole && k < (r < kRsRun ? m0 : m1)) store(row0 + (r < kRsRun ? 0 : m0) + k, t, v, part);
      }
    }
  }
  // (split) The sum of output `row`, whose CTAs' parts are at from[0], from[stride], ..
  __device__ __forceinline__ float combine(const float* from, size_t stride, int row) const {
    const int tile = RsShare::of(op.N, range.tiles, row), parts = cta_of((tile + 1) * per_tile - 1) - cta_of(tile * per_tile) + 1;
    float v = 0.0f;
#pragma unroll 4
    for (int i = 0; i < parts; ++i) v += __ldcg(from + i * stride);
    return v;
  }
  // kRsSum: warp w's sums of a tile that began before its share, in its ring.
  __device__ __forceinline__ float* held_area(int w) const {
    return reinterpret_cast<float*>(__cvta_shared_to_generic(ring + (w - (int)threadIdx.x / 32) * Z::WARP_RING));
  }

  // Of sum number j: the token's slot, the run, the row in it.
  __device__ __forceinline__ int token(int j) const { return kMma ? j / 4 % NT * 8 + lane % 4 * 2 + j % 2 : j; }
  __device__ __forceinline__ int run_of(int j) const { return kMma ? j / 2 % 2 : lane / kRsRun; }
  __device__ __forceinline__ int row_of(int j) const { return kMma ? j / (4 * NT) * 8 + lane / 4 : lane % kRsRun; }
};

}  // namespace moehub
