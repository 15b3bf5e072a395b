// smoe_mx_product: Y[slot] = W[idx[slot]] X[token of slot], both operands microscaled 4-bit floats, by the scaled matrix
// instructions (32 x 32 x 64, one e8m0 byte per 32 columns of a row, fp32 sums).
//   gemm     a work-group per tile of up to BT slots of one expert and BN weight rows; with few slots each finds its own among them
//   group    before it, with many slots: one work-group per expert lists the expert's slots, in order, and its tiles
#include "mx.hpp"
#include <type_traits>

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

#define MG_THREADS 1024
#define MG_MAX_SLOTS (1 << 22)

struct MxTile { int expert, count; };

struct MxGemmArgs {
  const uint8_t *wc, *ws, *xc, *xs;
  const int32_t* rows;        // slots, BT for every tile (behind a tile's last slot that slot again), or null: slot i is row i
  const MxTile* tiles;        // null without rows
  const int* n_tiles;
  const int32_t* idx;         // the slots' experts where the work-groups find their slots themselves, else null
  void* y;
  int E, N, K, n, k, x_slots, x_rows, swiglu, out_f32, col_tiles, super;
};

// Experts of the slots i .. i + 15 of a run that ends at i1 (i a multiple of four), all loads in flight at once; -1 behind the run.  An index outside the experts
// counts as the nearest of them.
#define MG_RUN 16
__device__ __forceinline__ void fetch_experts(const int32_t* idx, int i, int i1, int E, int (&v)[MG_RUN]) {
  int4 q[MG_RUN / 4];
#pragma unroll
  for (int u = 0; u < MG_RUN; u += 4) {
    q[u / 4] = make_int4(0, 0, 0, 0);
    if (i + u + 4 <= i1) q[u / 4] = *(const int4*)(idx + i + u);
    else {
      if (i + u < i1) q[u / 4].x = idx[i + u];
      if (i + u + 1 < i1) q[u / 4].y = idx[i + u + 1];
      if (i + u + 2 < i1) q[u / 4].z = idx[i + u + 2];
    }
  }
#pragma unroll
  for (int u = 0; u < MG_RUN; u++) {
    const int w = u % 4 == 0 ? q[u / 4].x : u % 4 == 1 ? q[u / 4].y : u % 4 == 2 ? q[u / 4].z : q[u / 4].w;
    v[u] = i + u < i1 ? max(0, min(w, E - 1)) : -1;
  }
}
__device__ __forceinline__ int wave_prefix(int v, int lane) {            // inclusive
  for (int s = 1; s < 64; s <<= 1) { const int o = __shfl_up(v, s); if (lane >= s) v += o; }
  return v;
}

// Work-group e: the slots of expert e, in order, to its tiles of bt.  Every work-group counts all slots, so that none waits
// for another.
//   Bound: one memory round trip and the launch; a thread's slots are fetched sixteen at a time before the first is used (one after the other: 9.9 us for
// 8192 slots, 60 experts).
__global__ __launch_bounds__(MG_THREADS) void mx_group_kernel(const int32_t* idx, int n, int E, int bt, int32_t* rows, MxTile* tiles, int* n_tiles) {
  __shared__ int count[SMOE_MAX_EXPERTS];
  __shared__ int wtot[MG_THREADS / 64];
  __shared__ int last;
  constexpr int RUN = MG_RUN;
  const int e = (int)blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid < SMOE_MAX_EXPERTS) count[tid] = 0;
  // every thread owns a contiguous run of slots, a multiple of four
  const int c = ((n + MG_THREADS - 1) / MG_THREADS + 3) & ~3, i0 = min(n, tid * c), i1 = min(n, i0 + c);
  int v[RUN];
  auto fetch = [&](int i) { fetch_experts(idx, i, i1, E, v); };
  fetch(i0);
  __syncthreads();
  int mine = 0;
  for (int i = i0; i < i1; i += RUN) {
    if (i != i0) fetch(i);
#pragma unroll
    for (int u = 0; u < RUN; u++)
      if (v[u] >= 0) { mine += v[u] == e; atomicAdd(&count[v[u]], 1); }
  }
  const int incl = wave_prefix(mine, lane);
  if (lane == 63) wtot[wave] = incl;
  __syncthreads();
  int t0 = 0;                                                           // tiles of the experts before e
  for (int f = lane; f < e; f += 64) t0 += (count[f] + bt - 1) / bt;
  for (int m = 32; m >= 1; m >>= 1) t0 += __shfl_xor(t0, m);
  int p = incl - mine;
#pragma unroll
  for (int w = 0; w < MG_THREADS / 64; w++) p += w < wave ? wtot[w] : 0;
  const int cnt = count[e], nt = (cnt + bt - 1) / bt;
  int32_t* out = rows + (size_t)t0 * bt;
  for (int i = i0; i < i1; i += RUN) {
    if (c > RUN) fetch(i);
#pragma unroll
    for (int u = 0; u < RUN; u++)
      if (v[u] == e) {
        out[p] = i + u;
        if (++p == cnt) last = i + u;
      }
  }
  __syncthreads();
  for (int r = cnt + tid; r < nt * bt; r += MG_THREADS) out[r] = last;      // (the expert's last slot fills its last tile)
  for (int i = tid; i < nt; i += MG_THREADS) tiles[t0 + i] = MxTile{e, min(bt, cnt - i * bt)};
  if (e == E - 1 && tid == 0) *n_tiles = t0 + nt;
}

__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ __forceinline__ u32x4 buffer_of(const void* base, uint32_t bytes) {
  const uint64_t v = (uint64_t)base;
  return u32x4{(uint32_t)uni((int)(uint32_t)v), (uint32_t)uni((int)(uint32_t)(v >> 32)) & 0xFFFFu, (uint32_t)uni((int)bytes), 0x00020000u};
}
// 16 or 4 bytes of every lane from memory straight into LDS: lane i's at lds + 16 i or 4 i.  The LDS address is an operand in M0, so the
// compiler writes that register (one wait state between the write and the load).  It does not count these loads.
__device__ __forceinline__ void to_lds16(u32x4 rsrc, uint32_t voff, uint32_t soff, uint32_t lds) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(voff), "s"(rsrc), "s"(soff), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ void to_lds4(u32x4 rsrc, uint32_t voff, uint32_t soff, uint32_t lds) {
  asm volatile("s_nop 0\n\tbuffer_load_dword %0, %1, %2 offen lds" ::"v"(voff), "s"(rsrc), "s"(soff), "{m0}"(lds) : "memory");
}

// Shape of a work-group: NT waves along the slots times NN along the weight rows, FT by FN fragments of 32 a wave.
//   A stage is 256 columns, 128 bytes of codes a row, brought straight into one of three buffers.  The eight 16-byte
// pieces of a row are stored permuted (piece p at p ^ (row / 2 % 8)), so that sixteen lanes of an operand read, sixteen rows of
// one piece, fall into different banks.  Half h of a wave multiplies blocks 4h .. 4h + 3 of a stage: its scales of
// a row are one dword, a byte per step.
//   What bounds it with many rows and long ones is the path from L2 to LDS: loads alone give 33 - 38 bytes a cycle and CU in pieces of 128 bytes on whole lines with 64 to 96 KB on
// their way, 22 (0.34 lines) in pieces of 64 bytes or where rows do not begin on lines (K not a multiple of 256).  4096 x 2048 x 10944 asks for 0.27 - 0.29 lines a cycle and CU, start
// and end counted in, with the matrix instructions busy a quarter of the time.
//   Scales come 16 bytes a row at a time, two stages' worth: a dword per stage would cost as many requests to L2 as half the codes (dense product,
// 4096 slots, N 2048, K 10944: 97 us with, 70 us without such loads).
template <int NT, int NN, int FT, int FN> struct MgShape {
  static constexpr int NW = NT * NN, BT = 32 * NT * FT, BN = 32 * NN * FN, ROWS = BT + BN, NBUF = 3;
  static constexpr int FRAGS = ROWS / 32, PAIRS = (FRAGS + 1) / 2;
  static constexpr int LCN = BN / 8 / NW, LCT = BT / 8 / NW, LC = LCN + LCT;      // code loads of a wave and stage
  static_assert(BN % (8 * NW) == 0 && BT % (8 * NW) == 0 && NW % 2 == 0 && PAIRS <= NW && BN % 64 == 0 && BT <= 64 * NW, "whole loads");
  static constexpr int codes = ROWS * 128, scales = PAIRS * 1024, extra = PAIRS * 256;      // a code buffer; one of two scale buffers; a fifth dword for each row
  static constexpr int chunk(bool unal) { return scales + (unal ? extra : 0); }
  static constexpr int slots_at(bool unal) { return NBUF * codes + 2 * chunk(unal); }       // where the tile's slots stand
  static constexpr int lds(bool unal) { return slots_at(unal) + BT * 4; }
  static constexpr int out_row = 128 + 16, out_wave = 32 * out_row;                         // result: a wave's place to turn its fragments round (16 bytes of padding keep the rows in different banks)
  static_assert(NW * out_wave <= NBUF * codes, "the results fit the code buffers");
};

// UNAL: a row's scales do not begin on a dword (K not a multiple of 128): a fifth dword is fetched, and scales are shifted.
template <class S, bool UNAL, int NT, int NN, int FT, int FN>
__device__ __forceinline__ void mx_gemm_tile(const MxGemmArgs& a, uint8_t* As) {
  constexpr int NW = S::NW, BT = S::BT, BN = S::BN, NBUF = S::NBUF, LC = S::LC, LCN = S::LCN, LCT = S::LCT;
  constexpr uint32_t STAGE = S::codes, SCALES = NBUF * STAGE, CHUNK = S::chunk(UNAL);
  constexpr uint32_t NONE = 0x80000000u;                               // beyond every buffer: nothing is fetched
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int c = lane & 31, h = lane >> 5;
  int* slots = (int*)(As + S::slots_at(UNAL));                          // the tile's slots
  // ---- how many tiles there are.  With a.idx: count the experts' slots and number their tiles (lane l: experts l, l + 64, ...)
  int *count = (int*)As, *wtot = count + SMOE_MAX_EXPERTS;             // (where the codes will be)
  const int run_len = ((a.n + 64 * NW - 1) / (64 * NW) + 3) & ~3, i0 = min(a.n, tid * run_len), i1 = min(a.n, i0 + run_len);
  int v[MG_RUN], cnt[SMOE_MAX_EXPERTS / 64], first[SMOE_MAX_EXPERTS / 64];
  int n_tiles = 0;
  if (a.idx) {
    fetch_experts(a.idx, i0, i1, a.E, v);
    for (int i = tid; i < SMOE_MAX_EXPERTS; i += 64 * NW) count[i] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MG_RUN; u++)
      if (v[u] >= 0) atomicAdd(&count[v[u]], 1);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < SMOE_MAX_EXPERTS / 64; q++) {
      const int x = lane + 64 * q;
      cnt[q] = count[x];
      first[q] = 0x7FFFFFFF;
      if (64 * q < a.E) {                                              // (uniform)
        const int t = (cnt[q] + BT - 1) / BT, sum = wave_prefix(t, lane);
        if (x < a.E) first[q] = n_tiles + sum - t;
        n_tiles += __builtin_amdgcn_readlane(sum, 63);
      }
    }
  } else {
    n_tiles = a.rows ? uni(*a.n_tiles) : (a.n + BT - 1) / BT;
  }
  // ---- which tile.  Consecutive items, `super` tiles of slots side by side for every tile of weight rows, stay on one XCD, whose L2 then serves the rows
  // they share
  const int n_items = n_tiles * a.col_tiles, run = (n_items + 7) >> 3;
  const int place = (int)blockIdx.x >> 3, item = ((int)blockIdx.x & 7) * run + place;
  if (place >= run || item >= n_items) return;
  const int per_band = a.super * a.col_tiles, band = uni(item / per_band), in_band = item - band * per_band;
  const int band_n = min(a.super, n_tiles - band * a.super), ct = uni(in_band / band_n), ti = band * a.super + in_band - ct * band_n;
  MxTile tile;
  if (a.idx) {
    // the last expert whose first tile is not past ti, and the slots of its rows m0 .. on
    int e = -1, m0 = 0, of = 0;
#pragma unroll
    for (int q = 0; q < SMOE_MAX_EXPERTS / 64; q++) e += (int)__builtin_popcountll(__ballot(first[q] <= ti));
    e = uni(e);
#pragma unroll
    for (int q = 0; q < SMOE_MAX_EXPERTS / 64; q++)
      if (q == e >> 6) {
        m0 = (ti - __builtin_amdgcn_readlane(first[q], e & 63)) * BT;
        of = __builtin_amdgcn_readlane(cnt[q], e & 63);
      }
    tile = MxTile{e, min(BT, of - m0)};
    int mine = 0;
#pragma unroll
    for (int u = 0; u < MG_RUN; u++) mine += v[u] == e;
    const int incl = wave_prefix(mine, lane);
    if (lane == 63) wtot[wave] = incl;
    __syncthreads();
    int p = incl - mine - m0;
#pragma unroll
    for (int w = 0; w < NW; w++) p += w < wave ? wtot[w] : 0;
#pragma unroll
    for (int u = 0; u < MG_RUN; u++)
      if (v[u] == e) {
        if (p >= 0 && p < BT) slots[p] = i0 + u;
        p++;
      }
    __syncthreads();
  } else {
    tile = a.rows ? a.tiles[ti] : MxTile{0, min(BT, a.n - ti * BT)};
    tile.expert = uni(tile.expert); tile.count = uni(tile.count);
    if (tid < BT) slots[tid] = a.rows ? a.rows[(size_t)ti * BT + tid] : ti * BT + min(tid, tile.count - 1);
  }
  const int nb = a.K >> 5, n0 = ct * BN, n_st = (nb + 7) >> 3, n_full = nb >> 3;
  const uint32_t rowb = (uint32_t)(a.K >> 1);
  const u32x4 rwc = buffer_of(a.wc + (size_t)tile.expert * a.N * rowb, (uint32_t)a.N * rowb);
  const u32x4 rws = buffer_of(a.ws + (size_t)tile.expert * a.N * nb, (uint32_t)a.N * (uint32_t)nb);
  const u32x4 rxc = buffer_of(a.xc, (uint32_t)a.x_rows * rowb);
  const u32x4 rxs = buffer_of(a.xs, ((uint32_t)a.x_rows * (uint32_t)nb + 3u) & ~3u);      // (whole dwords: every one fetched holds a byte of the array)
  // row of X of the tile's slot r; behind the last slot that slot again
  auto x_row = [&](int r) {
    const int rc = min(r, tile.count - 1);
    const int slot = a.idx ? slots[rc] : a.rows ? a.rows[(size_t)ti * BT + rc] : ti * BT + rc;
    return (uint32_t)(a.x_slots ? slot : slot / a.k);
  };
  // ---- addresses.  Code load q of a wave: rows 8 (NW q + wave) .. + 7 of the weight rows, then of the token rows; a lane's piece is the same for all q
  const int pr = lane >> 3, piece = (lane & 7) ^ (((8 * wave + pr) >> 1) & 7);
  const uint32_t wv = (uint32_t)(n0 + 8 * wave + pr) * rowb + piece * 16u;
  uint32_t xv[LCT];
#pragma unroll
  for (int q = 0; q < LCT; q++) xv[q] = x_row(8 * (NW * q + wave) + pr) * rowb + piece * 16u;
  const bool piece_last = (n_st - 1) * 8 + piece < nb;                 // the lane's piece exists in the last stage
  // scale loads: wave w brings fragments 2p and 2p + 1, p = w (or a copy of an earlier pair), a row a lane
  const int pair = wave % S::PAIRS, sf = 2 * pair + h;
  const bool of_w = pair < BN / 64;
  const uint32_t srow = of_w ? (uint32_t)min(n0 + sf * 32 + c, a.N - 1) : x_row(min(sf, S::FRAGS - 1) * 32 - BN + c);
  const uint32_t sv = srow * (uint32_t)nb;
  const u32x4 rs = of_w ? rws : rxs;
  const uint32_t as_base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)As;
  // code loads q0 .. q1 - 1 of the LC that bring stage st into a buffer (past the last stage nothing is fetched, but the load counts)
  auto issue = [&](int st, uint32_t buf, int q0, int q1) __attribute__((always_inline)) {
    const bool skip = st >= n_st || (st == n_st - 1 && !piece_last);
#pragma unroll
    for (int q = q0; q < q1; q++)
      to_lds16(q < LCN ? rwc : rxc, skip ? NONE : q < LCN ? wv + (uint32_t)(8 * NW * q) * rowb : xv[q < LCN ? 0 : q - LCN], (uint32_t)st * 128u, as_base + buf + (NW * q + wave) * 1024u);
  };
  constexpr int LSC = UNAL ? 2 : 1;
  // scales of stages 2g and 2g + 1.  A 16-byte load may run over the row's end (into the next row, or zeros behind the array)
  auto issue_scales = [&](int g) __attribute__((always_inline)) {
    const uint32_t lds = as_base + SCALES + (g & 1) * CHUNK;
    const int left = nb - 16 * g;                                      // the row's blocks from this chunk on
    to_lds16(rs, left <= 0 ? NONE : sv & ~3u, (uint32_t)g * 16u, lds + pair * 1024u);
    if (UNAL) to_lds4(rs, left + (int)(sv & 3u) <= 16 ? NONE : (sv & ~3u) + 16u, (uint32_t)g * 16u, lds + S::scales + pair * 256u);
  };
  const int wt = wave % NT, wn = wave / NT;
  f32x16 acc[FN][FT];
#pragma unroll
  for (int i = 0; i < FN; i++)
#pragma unroll
    for (int j = 0; j < FT; j++)
#pragma unroll
      for (int r = 0; r < 16; r++) acc[i][j][r] = 0.0f;
  // shift of an unaligned row's scales, in bytes
  uint32_t shw[FN], shx[FT];
#pragma unroll
  for (int i = 0; i < FN; i++) shw[i] = UNAL ? ((uint32_t)min(n0 + (wn * FN + i) * 32 + c, a.N - 1) * (uint32_t)nb) & 3u : 0u;
#pragma unroll
  for (int j = 0; j < FT; j++) shx[j] = UNAL ? (x_row((wt * FT + j) * 32 + c) * (uint32_t)nb) & 3u : 0u;
  // scales of fragment f, dword 2 (st % 2) + hh of the row's four
  auto scale_of = [&](int st, int f, int hh, uint32_t sh) __attribute__((always_inline)) {
    const uint8_t* at = As + SCALES + ((st >> 1) & 1) * CHUNK;
    const int d = 2 * (st & 1) + hh;
    const uint32_t o = f * 512 + c * 16 + d * 4;
    const uint32_t lo = *(const uint32_t*)(at + o);
    if (!UNAL) return lo;
    const uint32_t hi = *(const uint32_t*)(at + (d == 3 ? (uint32_t)(S::scales + f * 128 + c * 4) : o + 4));
    return (uint32_t)__builtin_amdgcn_alignbyte(hi, lo, sh);
  };
  auto read_scales = [&](int st, uint32_t (&sw)[FN], uint32_t (&sx)[FT]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FN; i++) sw[i] = scale_of(st, wn * FN + i, h, shw[i]);
#pragma unroll
    for (int j = 0; j < FT; j++) sx[j] = scale_of(st, BN / 32 + wt * FT + j, h, shx[j]);
  };
  struct Frags { u32x4 w[FN], x[FT]; };
  const uint32_t swz = (uint32_t)((c >> 1) & 7);
  auto read = [&](const uint8_t* st, int p, Frags& f) __attribute__((always_inline)) {
    const uint32_t o = c * 128 + (((uint32_t)p ^ swz) * 16);
#pragma unroll
    for (int i = 0; i < FN; i++) f.w[i] = *(const u32x4*)(st + (wn * FN + i) * 4096 + o);
#pragma unroll
    for (int j = 0; j < FT; j++) f.x[j] = *(const u32x4*)(st + (BN / 32 + wt * FT + j) * 4096 + o);
  };
  auto wide = [](u32x4 v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; };
  // one step: FN FT products of 64 columns; `extra(m)` follows product m
  auto mul = [&](auto s_c, const Frags& f, const uint32_t (&sw)[FN], const uint32_t (&sx)[FT], auto extra) __attribute__((always_inline)) {
    constexpr int s = decltype(s_c)::value;
#pragma unroll
    for (int i = 0; i < FN; i++)
#pragma unroll
      for (int j = 0; j < FT; j++) {
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(f.w[i]), wide(f.x[j]), acc[i][j], 4, 4, s, (int)sw[i], s, (int)sx[j]);
        extra(i * FT + j);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  const std::integral_constant<int, 0> s0{};
  const std::integral_constant<int, 1> s1{};
  const std::integral_constant<int, 2> s2{};
  const std::integral_constant<int, 3> s3{};
  // ---- columns.  The operands of a step are read while the one before it is multiplied.  In front of a stage's last step comes the barrier behind which the stage
  // has been read by all and the next one is there.  The loads into the buffer so freed are dealt to the products of the next four steps: a direct load keeps the texture
  // path busy for some 22 cycles, and eight waves that send all theirs at once stand still meanwhile.
  constexpr int M = FN * FT, HEAD = LC / 4;
  auto deal = [&](int st, uint32_t buf, int quarter, int m) __attribute__((always_inline)) {
    const int q0 = LC * quarter / 4, n = LC * (quarter + 1) / 4 - q0;
    issue(st, buf, q0 + n * m / M, q0 + n * (m + 1) / M);
  };
  issue_scales(0);
  issue_scales(1);
#pragma unroll
  for (int st = 0; st < NBUF - 1; st++) issue(st, st * STAGE, 0, LC);
  issue(NBUF - 1, (NBUF - 1) * STAGE, 0, HEAD);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LC + HEAD) : "memory");
  uint32_t cur = 0, before = (NBUF - 1) * STAGE;                       // buffer of the stage, and of the one before it
  uint32_t sw[FN], sx[FT];
  Frags f0, f1;
  if (n_full > 0) {
    read_scales(0, sw, sx);
    read(As, 4 * h, f0);
  }
  for (int st = 0; st < n_full; st++) {
    const uint8_t* at = As + cur;
    const uint32_t next = cur == (NBUF - 1) * STAGE ? 0 : cur + STAGE;
    const int ahead = st + NBUF - 1;
    read(at, 4 * h + 1, f1);
    __builtin_amdgcn_sched_barrier(0);
    mul(s0, f0, sw, sx, [&](int m) __attribute__((always_inline)) { deal(ahead, before, 1, m); });
    read(at, 4 * h + 2, f0);
    __builtin_amdgcn_sched_barrier(0);
    mul(s1, f1, sw, sx, [&](int m) __attribute__((always_inline)) { deal(ahead, before, 2, m); });
    read(at, 4 * h + 3, f1);
    __builtin_amdgcn_sched_barrier(0);
    mul(s2, f0, sw, sx, [&](int m) __attribute__((always_inline)) { deal(ahead, before, 3, m); });
    // younger than stage st + 1: a stage of codes and the scales sent for behind an odd stage
    if ((st & 1) == 0 && st > 0) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LC + LSC) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LC) : "memory");
    uint32_t nw[FN], nx[FT];
    read_scales(st + 1, nw, nx);                                       // (behind the last stage: what is read is not used)
    read(As + next, 4 * h, f0);
    __builtin_amdgcn_sched_barrier(0);
    mul(s3, f1, sw, sx, [&](int m) __attribute__((always_inline)) { deal(st + NBUF, cur, 0, m); });
    if (st & 1) issue_scales(((st + 1) >> 1) + 1);
#pragma unroll
    for (int i = 0; i < FN; i++) sw[i] = nw[i];
#pragma unroll
    for (int j = 0; j < FT; j++) sx[j] = nx[j];
    before = cur;
    cur = next;
  }
  if (n_full < n_st) {
    // the last blocks: half h takes `half` of them from h * half on; one that does not exist gets the scale 2^-127 on both sides,
    // and its products vanish (whatever codes LDS holds there)
    const uint8_t* at = As + cur;
    const int left = nb - n_full * 8, half = (left + 1) >> 1, mine = min(half, left - h * half);
    const uint32_t mask = mine >= 4 ? 0xFFFFFFFFu : (1u << (8 * max(mine, 0))) - 1u;
    auto pick = [&](int f, uint32_t sh) __attribute__((always_inline)) {
      const uint64_t v = ((uint64_t)scale_of(n_full, f, 1, sh) << 32) | scale_of(n_full, f, 0, sh);
      return (uint32_t)(v >> (8 * h * half)) & mask;
    };
#pragma unroll
    for (int i = 0; i < FN; i++) sw[i] = pick(wn * FN + i, shw[i]);
#pragma unroll
    for (int j = 0; j < FT; j++) sx[j] = pick(BN / 32 + wt * FT + j, shx[j]);
    for (int s = 0; s < half; s++) {
      Frags f;
      read(at, h * half + s, f);
      mul(s0, f, sw, sx, [](int) {});
#pragma unroll
      for (int i = 0; i < FN; i++) sw[i] >>= 8;
#pragma unroll
      for (int j = 0; j < FT; j++) sx[j] >>= 8;
    }
  }
  // (no load is on its way to LDS any more, and every wave has read its operands)
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  // ---- result.  Lane: slot c of a fragment, weight rows 8 (r / 4) + 4 h + r % 4.  A wave turns its fragments round in LDS of its own, so that it writes 64 or
  // 128 neighbouring bytes of a row of Y (32 with one fragment; stores of 4 or 8 bytes straight from the lanes: 22 of 96 us, 2048 tokens, top-4 of 60, N 2816, K 2048).
  const int osz = a.out_f32 ? 4 : 2, sg = a.swiglu;
  const int n_out = sg ? a.N >> 1 : a.N, per_pass = a.out_f32 && !sg ? 1 : FN;                     // columns of Y; fragments at a time
  const int lpr = 31 - __builtin_clz((unsigned)(per_pass * (sg ? 16 : 32) * osz / 16));           // log2 of a row's 16-byte pieces
  uint8_t* o = As + wave * S::out_wave;
  uint32_t low = 0;                                                    // lowest gate met, as bits: negative numbers are the larger the further they are from 0
  auto write = [&](auto far_c) __attribute__((always_inline)) {
    constexpr bool far = decltype(far_c)::value;
#pragma unroll
    for (int j = 0; j < FT; j++) {
      const int r0 = (wt * FT + j) * 32;
      if (r0 >= tile.count) continue;
#pragma unroll
      for (int i = 0; i < FN; i++) {
        const int ip = per_pass == 1 ? 0 : i;                            // place of the fragment in the pass
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const int nr = ip * 32 + 2 * r + 4 * h;
          const float v0 = acc[i][j][r], v1 = acc[i][j][r + 1], v2 = acc[i][j][r + 2], v3 = acc[i][j][r + 3];
          uint8_t* to = o + c * S::out_row;
          if (sg) {
            const float o0 = far ? swiglu(v0, v1) : swiglu_near(v0, v1), o1 = far ? swiglu(v2, v3) : swiglu_near(v2, v3);
            if (!far) low = max(max(low, __float_as_uint(v0)), __float_as_uint(v2));
            if (a.out_f32) *(float2*)(to + (nr >> 1) * 4) = make_float2(o0, o1);
            else *(uint32_t*)(to + (nr >> 1) * 2) = pack_bf16_rne(o0, o1);
          } else {
            if (a.out_f32) *(float4*)(to + nr * 4) = make_float4(v0, v1, v2, v3);
            else *(uint2*)(to + nr * 2) = make_uint2(pack_bf16_rne(v0, v1), pack_bf16_rne(v2, v3));
          }
        }
        if (ip == per_pass - 1) {
          asm volatile("" ::: "memory");                                 // (LDS keeps a wave's accesses in order; so does the compiler now)
          const int col0 = (n0 + (wn * FN + i - ip) * 32) >> sg;
          for (int x = lane; x < 32 << lpr; x += 64) {
            const int tr = x >> lpr, p = x & ((1 << lpr) - 1), col = col0 + p * (16 / osz);
            if (r0 + tr < tile.count && col < n_out)                     // (N is a multiple of 16: sixteen bytes are in or out)
              *(uint4*)((uint8_t*)a.y + ((size_t)slots[r0 + tr] * n_out + col) * osz) = *(const uint4*)(o + tr * S::out_row + p * 16);
          }
          asm volatile("" ::: "memory");
        }
      }
    }
  };
  // The shorter form of the SwiGLU for all; a wave that met a gate below -76, as good as none, writes its results once more.  2048 tokens, top-4 of 60,
  // N 2816, K 2048, on one machine each: 87.8 us against 87.1 with the shorter form alone; the longer form for all 89.2 against 83.2.
  write(std::false_type{});
  if (sg && __any(low > __float_as_uint(SWIGLU_FAR))) write(std::true_type{});
}

template <bool UNAL, int NT, int NN, int FT, int FN>
__global__ __launch_bounds__(64 * NT * NN) void mx_gemm_kernel(MxGemmArgs a) {
  extern __shared__ __align__(1024) uint8_t mdyn[];
  mx_gemm_tile<MgShape<NT, NN, FT, FN>, UNAL, NT, NN, FT, FN>(a, mdyn);
}

static inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// The tile shapes: slots, weight rows, work-groups that fit a CU, and a work-group's time with all of those filled, relative to the first shape's (dense,
// 4096 x 8192 x 8192: 320 / 214 / 162 us in 16 / 8 / 4 rounds).
struct MxShape { int bt, bn, per_cu; double cost; };
static const MxShape g_shapes[3] = {{32, 128, 2, 1.0}, {64, 128, 2, 1.34}, {128, 256, 1, 2.1}};
// tiles of bt slots: experts' last ones are taken to be half full
static long long likely_tiles(int n, int E, int bt) { return E == 1 ? (n + bt - 1) / bt : n / bt + (n < E ? n : E + 1) / 2; }
// The shape with the least rounds of work-groups times their cost; one round at least.  Microseconds of shapes 0 / 1 / 2 (top-6 of 64, N 2816, K 2048): 100
// tokens 39.0 / 39.3 / 45.3, 300 47.2 / 44.4 / 53.1, 800 75.8 / 61.9 / 66.6, 1500 118 / 87.7 / 82.2; dense, N 2048, K 2048: 256 rows 6.1 / 7.5 / 11.7, 4096 28.2 / 21.0 / 16.9.
static double rounds_of(const MxShape& s, int n, int E, int N) { return (double)likely_tiles(n, E, s.bt) * ((N + s.bn - 1) / s.bn) / (256.0 * s.per_cu); }      // (256 CUs, whatever the device has: smoe_mx_product_bytes, which has to decide alike, knows no device)
static int pick_shape(int n, int E, int N) {
  int best = 0;
  double least = 0.0;
  for (int i = 0; i < 3; i++) {
    const double rounds = rounds_of(g_shapes[i], n, E, N), t = (rounds > 1.0 ? rounds : 1.0) * g_shapes[i].cost;
    if (i == 0 || t < least) { best = i; least = t; }
  }
  return best;
}

template <bool UNAL, int NT, int NN, int FT, int FN>
static int launch_gemm_t(smoe_ctx* ctx, const MxGemmArgs& a, unsigned grid, int slot) {
  constexpr int lds = MgShape<NT, NN, FT, FN>::lds(UNAL);
  static_assert(lds <= 160 * 1024, "LDS");
  size_t& granted = ctx->mx_lds_granted[slot * 2 + UNAL];
  if (lds > 64 * 1024 && granted < (size_t)lds) {      // once per context: beyond the default 64 KB
    HIPCHK(ctx, hipFuncSetAttribute((const void*)mx_gemm_kernel<UNAL, NT, NN, FT, FN>, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    granted = lds;
  }
  mx_gemm_kernel<UNAL, NT, NN, FT, FN><<<grid, 64 * NT * NN, lds, ctx->stream>>>(a);
  HIPCHK(ctx, hipGetLastError());
  return SMOE_OK;
}
template <int NT, int NN, int FT, int FN>
static int launch_gemm(smoe_ctx* ctx, const MxGemmArgs& a, unsigned grid, int slot) {
  return (a.K >> 5) % 4 ? launch_gemm_t<true, NT, NN, FT, FN>(ctx, a, grid, slot) : launch_gemm_t<false, NT, NN, FT, FN>(ctx, a, grid, slot);
}

struct MxProductLayout { size_t rows, tiles, n_tiles, total; };
static int max_tiles_of(int n, int E, int bt) { return n / bt + (n < E ? n : E); }
static MxProductLayout product_layout(int T, int k, int E) {
  MxProductLayout l;
  const int n = T * k;
  size_t rows = 0, tiles = 0;
  for (const MxShape& s : g_shapes) {
    const size_t t = (size_t)max_tiles_of(n, E, s.bt);
    if (t * s.bt > rows) rows = t * s.bt;
    if (t > tiles) tiles = t;
  }
  l.rows = 0;
  l.tiles = up256(rows * 4);
  l.n_tiles = l.tiles + up256(tiles * sizeof(MxTile));
  l.total = l.n_tiles + 256;
  return l;
}

static int check_product(int E, int T, int k) {
  if (E <= 0 || E > SMOE_MAX_EXPERTS || T < 0 || k <= 0 || k > SMOE_MAX_TOPK || (long long)T * k > MG_MAX_SLOTS) return SMOE_ESHAPE;
  return SMOE_OK;
}

// Whether work-groups find their slots themselves: at most sixteen for a thread to look through, and at most two rounds of work-groups, each of which pays for
// the search what the list would cost all of them once and a launch.  Microseconds without / with a list (top-6 of 64, N 2816, K 2048): 32 tokens (1.6 rounds) 30.0 / 30.9, 100
// tokens (2.2) 41.0 / 39.0, 512 tokens (4.6) 56.3 / 53.5; 500 tokens, top-2 of 8, N 512, K 1024 (0.3) 7.3 / 9.7.
static bool searches_itself(int n, int E, int N, int shape) {
  const int waves[3] = {MgShape<1, 4, 1, 1>::NW, MgShape<2, 2, 1, 2>::NW, MgShape<2, 4, 2, 2>::NW};
  return n <= MG_RUN * 64 * waves[shape] && rounds_of(g_shapes[shape], n, E, N) <= 2.0;
}

extern "C" int smoe_mx_product_bytes(int T, int k, int E, int N, size_t* scratch_bytes) {
  if (!scratch_bytes) return SMOE_EINVAL;
  if (const int rc = check_product(E, T, k)) return rc;
  if (const int rc = check_mx_matrix(N, 32)) return rc;
  *scratch_bytes = T == 0 || searches_itself(T * k, E, N, pick_shape(T * k, E, N)) ? 0 : product_layout(T, k, E).total;
  return SMOE_OK;
}

extern "C" int smoe_mx_product(smoe_ctx* ctx, int E, int N, int K, const uint8_t* w_codes_dev, const uint8_t* w_scales_dev, int T, int k,
                               const uint8_t* x_codes_dev, const uint8_t* x_scales_dev, int x_slots, const int32_t* idx_dev, int swiglu, int out_dtype,
                               void* scratch_dev, size_t scratch_bytes, void* y_dev) {
  if (!ctx || (out_dtype != SMOE_F32 && out_dtype != SMOE_BF16) || (x_slots != 0 && x_slots != 1) || (swiglu != 0 && swiglu != 1)) return SMOE_EINVAL;
  if (const int rc = check_product(E, T, k)) return rc;
  if (const int rc = check_mx_matrix(N, K)) return rc;
  if (T == 0) return SMOE_OK;
  if ((long long)T * (x_slots ? k : 1) * (K / 2) >= (1ll << 31) || (long long)T * k * N > (1ll << 35) || (!idx_dev && (E != 1 || k != 1))) return SMOE_ESHAPE;
  const int n = T * k, shape = pick_shape(n, E, N);
  const bool lists = idx_dev && !searches_itself(n, E, N, shape);
  if (!w_codes_dev || !w_scales_dev || !x_codes_dev || !x_scales_dev || !y_dev || (lists && !scratch_dev)) return SMOE_EINVAL;
  if (!aligned16(w_codes_dev) || !aligned16(w_scales_dev) || !aligned16(x_codes_dev) || !aligned16(x_scales_dev) || !aligned16(idx_dev) ||
      !aligned16(y_dev) || !aligned16(scratch_dev))
    return SMOE_EALIGN;
  const MxProductLayout l = product_layout(T, k, E);
  if (lists && scratch_bytes < l.total) return SMOE_ESIZE;
  ON_DEVICE_OF(ctx);
  uint8_t* s = (uint8_t*)scratch_dev;
  MxGemmArgs a{w_codes_dev, w_scales_dev, x_codes_dev, x_scales_dev, nullptr, nullptr, nullptr, nullptr, y_dev, E, N, K, n, k, x_slots, T * (x_slots ? k : 1),
               swiglu, out_dtype == SMOE_F32, 0, 1};
  const int bt = g_shapes[shape].bt;
  a.col_tiles = (N + g_shapes[shape].bn - 1) / g_shapes[shape].bn;
  int max_tiles = (n + bt - 1) / bt;
  a.super = max_tiles / E < 1 ? 1 : max_tiles / E > 8 ? 8 : max_tiles / E;
  if (idx_dev) {
    max_tiles = max_tiles_of(n, E, bt);
    if (!lists) {
      a.idx = idx_dev;
    } else {
      int32_t* rows = (int32_t*)(s + l.rows);
      MxTile* tiles = (MxTile*)(s + l.tiles);
      int* n_tiles = (int*)(s + l.n_tiles);
      mx_group_kernel<<<E, MG_THREADS, 0, ctx->stream>>>(idx_dev, n, E, bt, rows, tiles, n_tiles);
      HIPCHK(ctx, hipGetLastError());
      a.rows = rows; a.tiles = tiles; a.n_tiles = n_tiles;
    }
  }
  const unsigned grid = ((unsigned)max_tiles * (unsigned)a.col_tiles + 7) / 8 * 8;
  if (shape == 0) return launch_gemm<1, 4, 1, 1>(ctx, a, grid, 0);
  if (shape == 1) return launch_gemm<2, 2, 1, 2>(ctx, a, grid, 1);
  return launch_gemm<2, 4, 2, 2>(ctx, a, grid, 2);
}
