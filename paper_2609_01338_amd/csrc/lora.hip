// Low-rank adapters of many requests beside a shared projection (gfx950):
//   y_r = base_r + s_a (x_r A_a^T) B_a^T,  a = adapter[r],
// with A_a [R][k] and B_a [n][R] f16 of which the first rank[a] ranks count.
//
// Two launches: the first forms t = x A^T, fp32, in K splits; the second adds
// the splits in order, scales them and adds t B^T to the rows.  The products
// of f16 x and A are exact and summed in fp32 (v_mfma_f32_16x16x32_f16); t
// stays fp32 and multiplies B, widened to fp32, on v_mfma_f32_16x16x4_f32, so
// no value on the way is rounded to f16 and y keeps the projection's
// precision.
//
// Memory-bound: a decode step reads each adapter once, a prefill its rows.
//  - Few rows (up to kGatherRows, any order): a workgroup per (group of up to
//    16 rows of one adapter, K split or column range), found by each
//    workgroup from the adapter list: row r begins a group when the rows
//    before it with its adapter fill whole groups.  Each adapter is read once
//    per 16 of its rows, however the rows are mixed.
//  - Many rows: tiles of 64 neighbouring rows; a tile with several adapters
//    runs once for each of them and keeps each row's own result.
// A row's results depend on no other row: a row is one column (or row) of an
// MFMA operand, and what other adapters make of it is dropped, not masked by
// zeros.
#include "mz_kernels.h"

namespace mzk {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kGatherRows = 512;     // rows up to which the adapter list is searched
constexpr int kTileRows = 64;
constexpr int kColsWg = 256;         // columns of a workgroup of the second product: 64 a wave

__device__ __forceinline__ bool has_adapter(const Lora& p, int a) { return (unsigned)a < (unsigned)p.n_adapters; }

__device__ __forceinline__ int rank_of(const Lora& p, int a) { return p.rank ? min(max(p.rank[a], 0), p.R) : p.R; }

// The group of rows that begins at row r (at most 16 rows with r's adapter):
// their indices in rows (LDS), written by every wave alike; the count, or 0
// where r begins none.
__device__ __forceinline__ int gather_group(const Lora& p, int r, int a, int* rows) {
  const int lane = threadIdx.x & 63;
  int v[kGatherRows / 64];
#pragma unroll
  for (int c = 0; c < kGatherRows / 64; ++c) {
    v[c] = -1;
    if (c * 64 < p.m) v[c] = p.adapter[min(c * 64 + lane, p.m - 1)];
  }
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
  int seen = 0, before = -1;       // rows of the adapter so far; those before r
#pragma unroll
  for (int c = 0; c < kGatherRows / 64; ++c) {
    if (c * 64 >= p.m) break;
    const bool match = c * 64 + lane < p.m && v[c] == a;
    const uint64_t mask = __ballot(match);
    if (r >> 6 == c) {
      before = seen + __popcll(mask & ((1ull << (r & 63)) - 1));
      if (before % 16) return 0;
    }
    if (before >= 0) {
      const int at = seen + __popcll(mask & below) - before;
      if (match && at >= 0 && at < 16) rows[at] = c * 64 + lane;
    }
    seen += __popcll(mask);
  }
  return min(seen - before, 16);
}

// acc += x A^T over the 32-wide K steps s0, s0 + ds, ... below s1: 16 rows x
// NR tiles of 16 ranks.  xr: this lane's x row, ar: its A row of rank tile 0
// (rank l % 16); the last step may pass k.
template <int NR>
__device__ __forceinline__ void shrink_steps(const Lora& p, const _Float16* xr, const _Float16* const (&ar)[NR], int s0,
                                             int s1, int ds, int n_rt, f32x4 (&acc)[NR]) {
  const int lg = (threadIdx.x & 63) >> 4;
#pragma unroll 4
  for (int s = s0; s < s1; s += ds) {
    const int k = s * 32 + lg * 8;
    const bool in = k < p.k;             // k is a multiple of 8
    const int kc = in ? k : 0;
    f16x8 xv = *reinterpret_cast<const f16x8*>(xr + kc);
    f16x8 av[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j)
      if (j < n_rt) av[j] = *reinterpret_cast<const f16x8*>(ar[j] + kc);
    if (!in) xv = f16x8{};
#pragma unroll
    for (int j = 0; j < NR; ++j)
      if (j < n_rt) {
        if (!in) av[j] = f16x8{};
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv, av[j], acc[j], 0, 0, 0);
      }
  }
}

// t [split][m][16 NR] of the K range of split blockIdx.y.
template <int NR, bool GATHER>
__global__ __launch_bounds__(256) void lora_shrink_kernel(Lora p) {
  constexpr int RP = 16 * NR;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, lg = lane >> 4;
  const int steps = (p.k + 31) / 32, ns = gridDim.y;
  const int s0 = (int)((int64_t)blockIdx.y * steps / ns), s1 = (int)((int64_t)(blockIdx.y + 1) * steps / ns);
  float* t = p.t + (int64_t)blockIdx.y * p.m * RP;
  const _Float16* ar[NR];
  f32x4 acc[NR];
  auto begin = [&](int a) {              // A rows of this lane; how many rank tiles count
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      ar[j] = p.a + ((int64_t)a * p.R + min(j * 16 + col, p.R - 1)) * p.k;
      acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  if constexpr (GATHER) {
    __shared__ int s_rows[16];
    __shared__ f32x4 s_acc[4][NR][64];
    const int r = blockIdx.x, a = __builtin_amdgcn_readfirstlane(p.adapter[r]);
    if (!has_adapter(p, a)) return;
    const int n = __builtin_amdgcn_readfirstlane(gather_group(p, r, a, s_rows));
    if (n == 0) return;
    __syncthreads();
    const int rank = rank_of(p, a), n_rt = (rank + 15) / 16;
    begin(a);
    // a quarter of the split's steps for each wave, in one run
    const int q0 = s0 + (s1 - s0) * w / 4, q1 = s0 + (s1 - s0) * (w + 1) / 4;
    shrink_steps<NR>(p, p.x + (int64_t)s_rows[min(col, n - 1)] * p.k, ar, q0, q1, 1, n_rt, acc);
#pragma unroll
    for (int j = 0; j < NR; ++j) s_acc[w][j][lane] = acc[j];
    __syncthreads();
    // wave w: rank tiles w, w + 4, ...; element e of lane l is row 4 (l / 16) + e, rank l % 16
    for (int j = w; j < NR; j += 4) {
      const f32x4 v = s_acc[0][j][lane] + s_acc[1][j][lane] + s_acc[2][j][lane] + s_acc[3][j][lane];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (lg * 4 + e < n) t[(int64_t)s_rows[lg * 4 + e] * RP + j * 16 + col] = j * 16 + col < rank ? v[e] : 0.f;
    }
  } else {
    // wave w: rows 16 w .. 16 w + 15 of the tile, over the whole split
    const int r0 = blockIdx.x * kTileRows + w * 16;
    if (r0 >= p.m) return;
    const int mine = r0 + col < p.m ? p.adapter[r0 + col] : -1;      // the same for the four lane groups
    uint64_t todo = __ballot(has_adapter(p, mine)) & 0xFFFF;
    while (todo) {
      const int a = __builtin_amdgcn_readlane(mine, __builtin_ctzll(todo));
      const uint64_t members = __ballot(mine == a) & 0xFFFF;
      todo &= ~members;
      const int rank = rank_of(p, a), n_rt = (rank + 15) / 16;
      begin(a);
      shrink_steps<NR>(p, p.x + (int64_t)min(r0 + col, p.m - 1) * p.k, ar, s0, s1, 1, n_rt, acc);
#pragma unroll
      for (int j = 0; j < NR; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if ((members >> (lg * 4 + e)) & 1)
            t[(int64_t)(r0 + lg * 4 + e) * RP + j * 16 + col] = j * 16 + col < rank ? acc[j][e] : 0.f;
    }
  }
}

// y of 16 NRT rows x 256 columns: wave w has columns 64 w .. 64 w + 63 of the
// range, as four tiles of 16.  The products run transposed, D[column][row], so
// that a lane holds four neighbouring columns of one row.
template <int NR, bool GATHER>
__global__ __launch_bounds__(256) void lora_expand_kernel(Lora p) {
  constexpr int RP = 16 * NR, PITCH = RP + 4, NRT = GATHER ? 1 : kTileRows / 16, ROWS = 16 * NRT;
  __shared__ int s_rows[16];
  __shared__ float s_t[ROWS][PITCH];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, lg = lane >> 4;
  const int c0 = blockIdx.y * kColsWg + w * 64;
  int n_rows, r0 = 0;
  if constexpr (GATHER) {
    const int r = blockIdx.x, a = __builtin_amdgcn_readfirstlane(p.adapter[r]);
    if (!has_adapter(p, a)) {            // such a row is the base's
      const int c = blockIdx.y * kColsWg + threadIdx.x;
      if (p.y != p.base && c < p.n) p.y[r * p.y_stride + c] = p.base[r * p.y_stride + c];
      return;
    }
    n_rows = __builtin_amdgcn_readfirstlane(gather_group(p, r, a, s_rows));
    if (n_rows == 0) return;
    __syncthreads();
  } else {
    r0 = blockIdx.x * ROWS;
    n_rows = min(ROWS, p.m - r0);
  }
  auto row_of = [&](int i) { return GATHER ? s_rows[i] : r0 + i; };
  // the base's values go out first; they are needed last
  f32x4 y[NRT][4];
  int rows[NRT], mine[NRT];
#pragma unroll
  for (int i = 0; i < NRT; ++i) {
    rows[i] = row_of(min(i * 16 + col, n_rows - 1));
    mine[i] = p.adapter[rows[i]];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int at = c0 + c * 16 + lg * 4;
      const float* b = p.base + (int64_t)rows[i] * p.y_stride + at;
      y[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (at + 4 <= p.n)
        y[i][c] = *reinterpret_cast<const f32x4*>(b);
      else
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (at + e < p.n) y[i][c][e] = b[e];
    }
  }
  // t of the rows: the splits added in order, times the row's scale
  for (int idx = threadIdx.x; idx < n_rows * (RP / 4); idx += 256) {
    const int i = idx / (RP / 4), j = (idx % (RP / 4)) * 4, r = row_of(i), a = p.adapter[r];
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
    if (has_adapter(p, a)) {
      const float* t = p.t + (int64_t)r * RP + j;
#pragma unroll 8
      for (int s = 0; s < p.n_split; ++s) v += *reinterpret_cast<const f32x4*>(t + (int64_t)s * p.m * RP);
      if (p.scale) v *= p.scale[a];
    }
    *reinterpret_cast<f32x4*>(&s_t[i][j]) = v;
  }
  __syncthreads();
  if (c0 >= p.n) return;
  f32x4 add[NRT][4];
#pragma unroll
  for (int i = 0; i < NRT; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) add[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int seen = GATHER ? mine[0] : (lane < n_rows ? p.adapter[r0 + lane] : -1);
  uint64_t todo = GATHER ? 1ull : __ballot(has_adapter(p, seen));
  while (todo) {
    const int a = __builtin_amdgcn_readlane(seen, __builtin_ctzll(todo));
    const uint64_t members = GATHER ? 1ull : __ballot(seen == a);
    todo &= ~members;
    const int rank = rank_of(p, a);
    f32x4 d[NRT][4];
#pragma unroll
    for (int i = 0; i < NRT; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) d[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NR; ++j) {
      if (j * 16 >= rank) break;
      // B of columns c0 + 16 c + l % 16, ranks 16 j + 4 (l / 16) .. + 3; ranks that do not count are zero
      const int k = j * 16 + lg * 4;
      f32x4 b[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int at = min(c0 + c * 16 + col, p.n - 1);
        const f16x4 v = *reinterpret_cast<const f16x4*>(p.b + ((int64_t)a * p.n + at) * p.R + (k < p.R ? k : 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) b[c][e] = k + e < rank ? (float)v[e] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < NRT; ++i) {
        if (!GATHER && !((members >> (i * 16)) & 0xFFFF)) continue;
        const f32x4 t = *reinterpret_cast<const f32x4*>(&s_t[i * 16 + col][k]);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) d[i][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[c][e], t[e], d[i][c], 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < NRT; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) add[i][c] = mine[i] == a ? d[i][c] : add[i][c];
  }
#pragma unroll
  for (int i = 0; i < NRT; ++i) {
    if (i * 16 + col >= n_rows) continue;
    const bool with = has_adapter(p, mine[i]);
    if (!with && p.y == p.base) continue;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int at = c0 + c * 16 + lg * 4;
      float* o = p.y + (int64_t)rows[i] * p.y_stride + at;
      const f32x4 v = with ? y[i][c] + add[i][c] : y[i][c];
      if (at + 4 <= p.n)
        *reinterpret_cast<f32x4*>(o) = v;
      else
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (at + e < p.n) o[e] = v[e];
    }
  }
}

int rank_tiles(int R) { return R <= 16 ? 1 : R <= 32 ? 2 : R <= 64 ? 4 : 8; }

template <int NR>
void launch_lora_nr(const Lora& p, hipStream_t s) {
  const int cols = (p.n + kColsWg - 1) / kColsWg;
  if (p.m <= kGatherRows) {
    hipLaunchKernelGGL((lora_shrink_kernel<NR, true>), dim3(p.m, p.n_split), dim3(256), 0, s, p);
    hipLaunchKernelGGL((lora_expand_kernel<NR, true>), dim3(p.m, cols), dim3(256), 0, s, p);
  } else {
    const int tiles = (p.m + kTileRows - 1) / kTileRows;
    hipLaunchKernelGGL((lora_shrink_kernel<NR, false>), dim3(tiles, p.n_split), dim3(256), 0, s, p);
    hipLaunchKernelGGL((lora_expand_kernel<NR, false>), dim3(tiles, cols), dim3(256), 0, s, p);
  }
}

}  // namespace

// K splits: enough workgroups for the chip, at least two steps of 32 a wave.
int lora_splits(int m, int k) {
  const int steps = (k + 31) / 32;
  const int tiles = m <= kGatherRows ? m : (m + kTileRows - 1) / kTileRows;
  const int want = m <= kGatherRows ? 1024 / tiles : 512 / tiles;
  const int most = m <= kGatherRows ? steps / 8 : steps / 8;
  const int ns = want < most ? want : most;
  return ns < 1 ? 1 : ns > 16 ? 16 : ns;
}

int64_t lora_ws_bytes(int m, int k, int R) { return (int64_t)lora_splits(m, k) * m * rank_tiles(R) * 16 * 4; }

void launch_lora(Lora p, void* ws, hipStream_t s) {
  p.t = reinterpret_cast<float*>(ws);
  p.n_split = lora_splits(p.m, p.k);
  switch (rank_tiles(p.R)) {
    case 1: launch_lora_nr<1>(p, s); break;
    case 2: launch_lora_nr<2>(p, s); break;
    case 4: launch_lora_nr<4>(p, s); break;
    default: launch_lora_nr<8>(p, s); break;
  }
}

}  // namespace mzk
