// smoe_mx_product: Y[slot] = W[idx[slot]] X[token of slot], both operands microscaled 4-bit floats, by the scaled matrix
// instructions (32 x 32 x 64, one e8m0 byte per 32 columns of a row, fp32 sums).
//   group    one work-group per expert: the expert's slots, in order, and its tiles of at most BT of them
//   gemm     a work-group per tile of slots and BN weight rows
#include "mx.hpp"

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

#define MG_THREADS 1024
#define MG_MAX_SLOTS (1 << 22)

struct MxTile { int expert, first, count, pad; };

struct MxGemmArgs {
  const uint8_t *wc, *ws, *xc, *xs;
  const int32_t* rows;        // slots sorted by expert, or null: slot i is row i
  const MxTile* tiles;        // null without rows
  const int* n_tiles;
  void* y;
  int N, K, n, k, x_slots, col_tiles;
};

// Work-group e: slots of expert e to rows[], its tiles to tiles[].  Every work-group counts all slots, so that none waits
// for another.  An index outside the experts counts as the nearest of them.
__global__ __launch_bounds__(MG_THREADS) void mx_group_kernel(const int32_t* idx, int n, int E, int bt, int32_t* rows, MxTile* tiles, int* n_tiles) {
  __shared__ int count[SMOE_MAX_EXPERTS];
  __shared__ int wtot[MG_THREADS / 64];
  const int e = (int)blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid < SMOE_MAX_EXPERTS) count[tid] = 0;
  __syncthreads();
  const int c = (n + MG_THREADS - 1) / MG_THREADS, i0 = min(n, tid * c), i1 = min(n, i0 + c);
  auto expert = [&](int i) { const int v = idx[i]; return v < 0 ? 0 : v >= E ? E - 1 : v; };
  int mine = 0;
  for (int i = i0; i < i1; i++) {
    const int v = expert(i);
    mine += v == e;
    atomicAdd(&count[v], 1);
  }
  int incl = mine;
  for (int s = 1; s < 64; s <<= 1) { const int o = __shfl_up(incl, s); if (lane >= s) incl += o; }
  if (lane == 63) wtot[wave] = incl;
  __syncthreads();
  int before = 0, tiles_before = 0;
  for (int f = lane; f < e; f += 64) { before += count[f]; tiles_before += (count[f] + bt - 1) / bt; }
  for (int m = 32; m >= 1; m >>= 1) { before += __shfl_xor(before, m); tiles_before += __shfl_xor(tiles_before, m); }
  int p = before + incl - mine;
  for (int w = 0; w < wave; w++) p += wtot[w];
  for (int i = i0; i < i1; i++)
    if (expert(i) == e) rows[p++] = i;
  const int cnt = count[e], nt = (cnt + bt - 1) / bt;
  for (int i = tid; i < nt; i += MG_THREADS) tiles[tiles_before + i] = MxTile{e, before + i * bt, min(bt, cnt - i * bt), 0};
  if (e == E - 1 && tid == 0) *n_tiles = tiles_before + nt;
}

template <int OUT> __device__ __forceinline__ void store1(void* p, size_t i, float v) {
  if (OUT == SMOE_F32) ((float*)p)[i] = v;
  else ((__bf16*)p)[i] = (__bf16)v;
}

// Four waves side by side over the weight rows; a wave 64 slots by 64 weight rows.
template <int OUT, int SWIGLU>
__global__ __launch_bounds__(256) void mx_gemm_kernel(MxGemmArgs a) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = lane & 31, h = lane >> 5;
  const int ti = (int)blockIdx.x / a.col_tiles, ct = (int)blockIdx.x % a.col_tiles;
  MxTile tile;
  if (a.rows) {
    if (ti >= *a.n_tiles) return;
    tile = a.tiles[ti];
  } else {
    tile = MxTile{0, ti * 64, min(64, a.n - ti * 64), 0};
  }
  const int nb = a.K >> 5, n0 = ct * 256 + wave * 64;
  if (n0 >= a.N) return;
  const uint8_t *wc[2], *ws[2], *xc[2], *xs[2];
#pragma unroll
  for (int f = 0; f < 2; f++) {
    const size_t wr = (size_t)tile.expert * a.N + min(n0 + f * 32 + c, a.N - 1);
    const int i = tile.first + min(f * 32 + c, tile.count - 1);
    const int slot = a.rows ? a.rows[i] : i;
    const size_t xr = a.x_slots ? slot : slot / a.k;
    wc[f] = a.wc + wr * (size_t)(a.K >> 1); ws[f] = a.ws + wr * (size_t)nb;
    xc[f] = a.xc + xr * (size_t)(a.K >> 1); xs[f] = a.xs + xr * (size_t)nb;
  }
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; i++)
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int r = 0; r < 16; r++) acc[i][j][r] = 0.0f;
  for (int b0 = 0; b0 < nb; b0 += 2) {
    const int b = b0 + h, bc = min(b, nb - 1);
    i32x8 w[2], x[2];
    int sw[2], sx[2];
#pragma unroll
    for (int f = 0; f < 2; f++) {
      const u32x4 cw = *(const u32x4*)(wc[f] + (size_t)bc * 16), cx = *(const u32x4*)(xc[f] + (size_t)bc * 16);
      w[f] = i32x8{(int)cw[0], (int)cw[1], (int)cw[2], (int)cw[3], 0, 0, 0, 0};
      x[f] = i32x8{(int)cx[0], (int)cx[1], (int)cx[2], (int)cx[3], 0, 0, 0, 0};
      // past the last block: both scales 2^-127, the products vanish
      sw[f] = b < nb ? ws[f][bc] : 0;
      sx[f] = b < nb ? xs[f][bc] : 0;
    }
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int j = 0; j < 2; j++) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[i], x[j], acc[i][j], 4, 4, 0, sw[i], 0, sx[j]);
  }
  // lane: slot c of the fragment, weight rows 8 (r / 4) + 4 h + r % 4
#pragma unroll
  for (int j = 0; j < 2; j++) {
    if (j * 32 + c >= tile.count) continue;
    const int at = tile.first + j * 32 + c;
    const size_t slot = a.rows ? a.rows[at] : at;
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const int nr = n0 + i * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
        if (nr >= a.N) continue;
        const float v0 = acc[i][j][r], v1 = acc[i][j][r + 1];
        if (SWIGLU) {
          store1<OUT>(a.y, slot * (size_t)(a.N >> 1) + (nr >> 1), v0 / (1.0f + expf(-v0)) * v1);
        } else {
          store1<OUT>(a.y, slot * (size_t)a.N + nr, v0);
          store1<OUT>(a.y, slot * (size_t)a.N + nr + 1, v1);
        }
      }
  }
}

static inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

struct MxProductLayout { size_t rows, tiles, n_tiles, total; };
static MxProductLayout product_layout(int T, int k, int E) {
  MxProductLayout l;
  const size_t n = (size_t)T * k;
  l.rows = 0;
  l.tiles = up256(n * 4);
  l.n_tiles = l.tiles + up256((n / 32 + (size_t)E) * sizeof(MxTile));
  l.total = l.n_tiles + 256;
  return l;
}

static int check_product(int E, int T, int k) {
  if (E <= 0 || E > SMOE_MAX_EXPERTS || T < 0 || k <= 0 || k > SMOE_MAX_TOPK || (long long)T * k > MG_MAX_SLOTS) return SMOE_ESHAPE;
  return SMOE_OK;
}

extern "C" int smoe_mx_product_bytes(int T, int k, int E, size_t* scratch_bytes) {
  if (!scratch_bytes) return SMOE_EINVAL;
  if (const int rc = check_product(E, T, k)) return rc;
  *scratch_bytes = product_layout(T, k, E).total;
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
  if (!w_codes_dev || !w_scales_dev || !x_codes_dev || !x_scales_dev || !y_dev || (idx_dev && !scratch_dev)) return SMOE_EINVAL;
  if (!aligned16(w_codes_dev) || !aligned16(w_scales_dev) || !aligned16(x_codes_dev) || !aligned16(x_scales_dev) || !aligned16(idx_dev) ||
      !aligned16(y_dev) || !aligned16(scratch_dev))
    return SMOE_EALIGN;
  const MxProductLayout l = product_layout(T, k, E);
  if (idx_dev && scratch_bytes < l.total) return SMOE_ESIZE;
  ON_DEVICE_OF(ctx);
  const int n = T * k, bt = 64;
  uint8_t* s = (uint8_t*)scratch_dev;
  MxGemmArgs a{w_codes_dev, w_scales_dev, x_codes_dev, x_scales_dev, nullptr, nullptr, nullptr, y_dev, N, K, n, k, x_slots, (N + 255) / 256};
  int max_tiles = (n + bt - 1) / bt;
  if (idx_dev) {
    int32_t* rows = (int32_t*)(s + l.rows);
    MxTile* tiles = (MxTile*)(s + l.tiles);
    int* n_tiles = (int*)(s + l.n_tiles);
    mx_group_kernel<<<E, MG_THREADS, 0, ctx->stream>>>(idx_dev, n, E, bt, rows, tiles, n_tiles);
    HIPCHK(ctx, hipGetLastError());
    a.rows = rows; a.tiles = tiles; a.n_tiles = n_tiles;
    max_tiles = n / bt + (n < E ? n : E);
  }
  const unsigned grid = (unsigned)max_tiles * (unsigned)a.col_tiles;
  if (out_dtype == SMOE_F32) {
    if (swiglu) mx_gemm_kernel<SMOE_F32, 1><<<grid, 256, 0, ctx->stream>>>(a);
    else mx_gemm_kernel<SMOE_F32, 0><<<grid, 256, 0, ctx->stream>>>(a);
  } else {
    if (swiglu) mx_gemm_kernel<SMOE_BF16, 1><<<grid, 256, 0, ctx->stream>>>(a);
    else mx_gemm_kernel<SMOE_BF16, 0><<<grid, 256, 0, ctx->stream>>>(a);
  }
  HIPCHK(ctx, hipGetLastError());
  return SMOE_OK;
}
