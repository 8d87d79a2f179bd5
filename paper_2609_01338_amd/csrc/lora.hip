// Low-rank adapters of many requests beside a shared projection (gfx950):
//   y_r = base_r + s_a (x_r A_a^T) B_a^T,  a = adapter[r],
// with A_a [R][k] and B_a [n][R] f16 of which the first rank[a] ranks count.
//
// Two steps: the first forms t = x A^T, fp32, in K splits; the second adds
// the splits in order and adds s (t B^T) to the rows.  The products of f16 x and
// A are exact and summed in fp32 (v_mfma_f32_16x16x32_f16).  For the second
// product t is cut into three bf16 values of 8 bits each and B into two (8 and 3
// bits), both exactly and whatever their size: the six products of the parts are
// exact too (v_mfma_f32_16x16x32_bf16), so nothing of t or B is lost, also where
// a small t meets a large B, in 3/8 of the time of the fp32 matrix instructions.
// The scale comes last, in one rounding with the base.
//
// Memory-bound: a decode step reads each adapter once, a prefill its rows.
// Measured: 1 row of 2048 x 2048, rank 16, 5.6 us, latency; 33 rows over 24
// adapters, 4096 x 4096, rank 32, 4.5 + 5.9, two chains of dependent loads (list,
// rows, x and A; then list, t, B, base); 4099 rows over 6, rank 64, 18.5 + 43.7:
// 171 MB at 2.7 TB/s.
//  - Few rows (up to kGatherRows): a workgroup per (group of up to 16 rows of
//    one adapter, K split or column range), found by each workgroup from the
//    adapter list: row r begins a group when the rows before it with its
//    adapter fill whole groups.
//  - Many rows: tiles of up to 64 rows of one adapter.  The workgroups of the
//    first product count the adapter list and pick their tile's rows out of
//    it, and leave the tiles to the second.  More than kPlanRows rows run as
//    several such calls.
//  Either way rows may be mixed as they like: an adapter is read once per 16
//  (64) of its rows.
// A row's results depend on no other row: a row is one column (or row) of an
// MFMA operand, and what other adapters make of it is dropped, not masked by
// zeros.
#include "mz_kernels.h"

namespace mzk {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4), aligned(4)));      // the adapter list begins anywhere
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

// Rows up to which groups are searched.  Groups against tiles, measured in a
// graph, 4096 x 4096 of rank 16: 33 rows of one adapter 9.9 against 11.7 us,
// with an adapter each 9.6 against 17.8; 64 rows 12.4 against 12.3, over 8 mixed
// adapters 9.0 against 12.2, with an adapter each 11.7 against 25.6.  4096 x
// 14336, rank 32, 64 rows: 21.5 against 16.1, 10.5 against 18.5, 25.8 against
// 58.4.  At 128 rows the first kind is nearly twice as slow.
constexpr int kGatherRows = 64;
constexpr int kPlanRows = 8192;      // rows of a call whose tiles are counted: 32 entries a thread
constexpr int kTile = 64;            // rows of a tile
constexpr int kColsWg = 256;         // columns of a workgroup of few rows' second product: 64 a wave
constexpr int kColsFused = 128;      // the same where one launch does both: 32 a wave

__device__ __forceinline__ bool has_adapter(const Lora& p, int a) { return (unsigned)a < (unsigned)p.n_adapters; }

__device__ __forceinline__ int rank_of(const Lora& p, int a) { return p.rank ? min(max(p.rank[a], 0), p.R) : p.R; }

// The group of rows that begins at row r (at most 16 rows with r's adapter):
// their indices in rows (LDS), written by every wave alike; the count, or 0
// where r begins none.
__device__ __forceinline__ int gather_group(const Lora& p, int r, int a, int* rows) {
  const int lane = threadIdx.x & 63;
  static_assert(kGatherRows == 64, "a row a lane");
  const bool match = lane < p.m && p.adapter[min(lane, p.m - 1)] == a;
  const uint64_t mask = __ballot(match);
  const int before = __popcll(mask & ((1ull << r) - 1));
  if (before % 16) return 0;
  const int at = __popcll(mask & ((1ull << lane) - 1)) - before;
  if (match && at >= 0 && at < 16) rows[at] = lane;
  return min(__popcll(mask) - before, 16);
}

// LDS of plan_tile: the call's adapters, where the adapter changes (or a window
// of 64 rows begins), how many rows each adapter has.
struct PlanLds {
  uint16_t list[kPlanRows];
  uint8_t change[kPlanRows / 4];         // bit e: row 4 i + e
  int hist[kLoraAdapters + 1];
};

// Runs of one adapter, each within a window of 64 rows, that make the tiles as
// they stand; with more of them the rows are sorted.  As they stand against
// sorted, 4096 rows of 4096 x 4096, rank 64 (16): runs of 64 rows (as many as
// windows) 50.9 (38.9) against 64.0 (51.8) us, of 100 (1.6 a window) 64.9
// (49.1) against 75.9 (58.2), of 48 (2) 70.8 (54.4) against 68.0 (52.2), of 24
// (3.3) 104 (78) against 67 (51).  The eight more are for few rows, whose tiles do
// not fill the chip either way: 128 rows in 8 runs 15.6 (11.7) against 17.0 (13.3),
// 256 in 8 17.0 (12.6) against 17.5 (13.7); near the rule's end ranks decide: 256
// rows in 13 runs 19.7 (13.7) against 18.0 (13.9), 512 in 19 23.5 (17.3) against
// 22.4 (15.8).
__host__ __device__ inline int most_runs(int m) {
  const int windows = (m + 63) / 64;
  return windows + windows * 3 / 4 + 8;
}

// Four nibbles, one a byte, together.
__device__ __forceinline__ uint64_t sixteen(uint32_t d) {
  const uint32_t x = d | d >> 4;
  return (x & 0xff) | (x >> 8 & 0xff00);
}

// The rows of tile `tile`, of one adapter (p.n_adapters: none): the adapter,
// the rows (LDS, written up to the count) and the count, 0 where there is no
// such tile.  Where rows of one adapter follow each other (prompts), the runs
// within windows of 64 rows are the tiles.  Else the rows are taken as sorted
// by adapter, each adapter's in their order and in tiles of their own: counted
// in LDS, then the tile's picked by their rank.  Every thread of 256 takes
// part, and every workgroup comes to the same tiles.  (The sort's loops over
// the list are kept short: unrolled, their code took longer to fetch than to
// run.)
__device__ __forceinline__ int plan_tile(const Lora& p, int tile, PlanLds& s, int* rows, int& adapter) {
  __shared__ int s_red[4], s_found[2];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int buckets = p.n_adapters + 1, chunks = (p.m + 255) / 256;  // 64-row chunks of a wave
  const int r0 = w * chunks * 64, r1 = min(r0 + chunks * 64, p.m);   // this wave's rows
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
  constexpr int AHEAD = kPlanRows / 1024;    // 16 bytes of the list a thread each: all of it in one trip
  i32x4 v[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int r = 1024 * i + 4 * (int)threadIdx.x;
    if (1024 * i >= p.m) break;
    if (r + 4 <= p.m) {
      v[i] = *reinterpret_cast<const i32x4*>(p.adapter + r);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = r + e < p.m ? p.adapter[r + e] : -1;
    }
  }
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int r = 1024 * i + 4 * (int)threadIdx.x;
    if (1024 * i >= p.m) break;
    u16x4 mine;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine[e] = (uint16_t)(has_adapter(p, v[i][e]) ? v[i][e] : p.n_adapters);
    int prev = __shfl_up((int)mine[3], 1), change = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (r + e < p.m && ((r + e) % 64 == 0 || mine[e] != prev)) change |= 1 << e;
      prev = mine[e];
    }
    *reinterpret_cast<u16x4*>(&s.list[r]) = mine;
    s.change[r / 4] = (uint8_t)change;
  }
  if (threadIdx.x == 0) s_found[0] = -1;
  __syncthreads();
  {  // lane l: windows 2 l and 2 l + 1
    static_assert(kPlanRows / 64 == 128, "windows of a wave's lanes");
    uint64_t change[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      change[i] = 0;
      if ((2 * lane + i) * 64 >= p.m) continue;
      const uint4 d = *reinterpret_cast<const uint4*>(&s.change[(2 * lane + i) * 16]);
      change[i] = sixteen(d.x) | sixteen(d.y) << 16 | sixteen(d.z) << 32 | sixteen(d.w) << 48;
    }
    const int c0 = __popcll(change[0]), c1 = __popcll(change[1]);
    int sum = c0 + c1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(sum, o);
      if (lane >= o) sum += u;
    }
    const int total = __builtin_amdgcn_readlane(sum, 63);
    if (total <= most_runs(p.m)) {
      if (tile >= total) return 0;
      const int first = sum - c0 - c1;
      const int l = __builtin_ctzll(__ballot(tile < sum));         // the first window pair that ends past the tile
      int nth = tile - __builtin_amdgcn_readlane(first, l), window = 2 * l;
      const int in_first = __builtin_amdgcn_readlane(c0, l);
      uint64_t starts = change[0];
      if (nth >= in_first) {
        nth -= in_first;
        ++window;
        starts = change[1];
      }
      starts = (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(starts >> 32), l) << 32 |
               (unsigned)__builtin_amdgcn_readlane((int)starts, l);
      for (; nth > 0; --nth) starts &= starts - 1;
      const int start = __builtin_ctzll(starts);
      starts &= starts - 1;
      const int r = window * 64 + start, end = min(window * 64 + (starts ? (int)__builtin_ctzll(starts) : 64), p.m);
      adapter = __builtin_amdgcn_readfirstlane(s.list[r]);
      if (threadIdx.x < 64 && r + lane < end) rows[lane] = r + lane;
      __syncthreads();
      return end - r;
    }
  }
  for (int i = threadIdx.x; i < buckets; i += 256) s.hist[i] = 0;
  __syncthreads();
#pragma unroll 2
  for (int r = r0; r < r1; r += 64)
    if (r + lane < r1) atomicAdd(&s.hist[s.list[r + lane]], 1);
  __syncthreads();
  int before = 0;
#pragma unroll 1
  for (int b0 = 0; b0 < buckets; b0 += 256) {
    const int b = b0 + threadIdx.x, mine = b < buckets ? (s.hist[b] + kTile - 1) / kTile : 0;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(sum, o);
      if (lane >= o) sum += u;
    }
    __syncthreads();
    if (lane == 63) s_red[w] = sum;
    __syncthreads();
    int first = before + sum - mine;
    for (int i = 0; i < w; ++i) first += s_red[i];
    if (tile >= first && tile < first + mine) {
      s_found[0] = b;
      s_found[1] = (tile - first) * kTile;
    }
    before += s_red[0] + s_red[1] + s_red[2] + s_red[3];
    if (tile < before) break;
  }
  __syncthreads();
  adapter = __builtin_amdgcn_readfirstlane(s_found[0]);
  if (adapter < 0) return 0;
  const int begin = s_found[1], n = min(s.hist[adapter] - begin, kTile);
  int count = 0;                       // of the adapter's rows among this wave's
#pragma unroll 1
  for (int r = r0; r < r1; r += 64) count += __popcll(__ballot(r + lane < r1 && s.list[r + lane] == adapter));
  __syncthreads();
  if (lane == 0) s_red[w] = count;
  __syncthreads();
  int rank = 0;                        // rows of the adapter before this wave's
  for (int i = 0; i < w; ++i) rank += s_red[i];
#pragma unroll 1
  for (int r = r0; r < r1 && rank < begin + kTile; r += 64) {
    const bool is = r + lane < r1 && s.list[r + lane] == adapter;
    const uint64_t same = __ballot(is);
    const int at = rank + __popcll(same & below) - begin;
    if (is && at >= 0 && at < kTile) rows[at] = r + lane;
    rank += __popcll(same);
  }
  __syncthreads();
  return n;
}

// acc += x A^T over the 32-wide K steps s0 .. s1 - 1 of 16 rows and NT tiles
// of 16 ranks.  xr: this lane's x row, ar: its A row (rank l % 16 of each
// tile).  No branch lies between the loads of a few steps, so all of them are
// in flight together; the last step may pass k.
template <int NT, int NR>
__device__ __forceinline__ void shrink_steps(int k_all, const _Float16* xr, const _Float16* const (&ar)[NR], int s0, int s1,
                                             f32x4 (&acc)[NR]) {
  const int lg = (threadIdx.x & 63) >> 4;
  const int full = min(s1, k_all / 32);
  constexpr int U = 4;
  int s = s0;
  for (; s + U <= full; s += U) {
    f16x8 xv[U], av[U][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = (s + u) * 32 + lg * 8;
      xv[u] = *reinterpret_cast<const f16x8*>(xr + k);
#pragma unroll
      for (int j = 0; j < NT; ++j) av[u][j] = *reinterpret_cast<const f16x8*>(ar[j] + k);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv[u], av[u][j], acc[j], 0, 0, 0);
  }
  for (; s < s1; ++s) {
    const int k = s * 32 + lg * 8;
    const bool in = k < k_all;             // k_all is a multiple of 8
    const f16x8 xv = *reinterpret_cast<const f16x8*>(xr + (in ? k : 0));
    f16x8 av[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) av[j] = *reinterpret_cast<const f16x8*>(ar[j] + (in ? k : 0));
#pragma unroll
    for (int j = 0; j < NT; ++j)
      acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(in ? xv : f16x8{}, in ? av[j] : f16x8{}, acc[j], 0, 0, 0);
  }
}

// x A^T of the group's n rows over the steps s0 .. s1 - 1: a quarter of them
// for each of the four waves, joined through LDS; wave w then has the rank
// tiles w, w + 4, ... in v, element e of lane l being row 4 (l / 16) + e,
// rank l % 16 of the tile.
template <int NR>
__device__ __forceinline__ void shrink_group(const Lora& p, int a, int rank, int n, const int* s_rows, int s0, int s1,
                                             f32x4 (&s_acc)[4][NR][64], f32x4 (&v)[(NR + 3) / 4]) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15;
  const int q0 = s0 + (s1 - s0) * w / 4, q1 = s0 + (s1 - s0) * (w + 1) / 4;
  const int n_rt = (rank + 15) / 16;
  const _Float16 *ar[NR], *xr = p.x + (int64_t)s_rows[min(col, n - 1)] * p.k;
  f32x4 acc[NR];
#pragma unroll
  for (int j = 0; j < NR; ++j) {
    ar[j] = p.a + ((int64_t)a * p.R + max(min(j * 16 + col, rank - 1), 0)) * p.k;
    acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // rank tiles past the rank are left out, by powers of two
  if (n_rt <= 1) shrink_steps<1>(p.k, xr, ar, q0, q1, acc);
  else if (NR == 2 || (NR > 2 && n_rt <= 2)) shrink_steps<NR >= 2 ? 2 : 1>(p.k, xr, ar, q0, q1, acc);
  else if (NR == 4 || (NR > 4 && n_rt <= 4)) shrink_steps<NR >= 4 ? 4 : 1>(p.k, xr, ar, q0, q1, acc);
  else shrink_steps<NR>(p.k, xr, ar, q0, q1, acc);
#pragma unroll
  for (int j = 0; j < NR; ++j) s_acc[w][j][lane] = acc[j];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < (NR + 3) / 4; ++i) {
    const int j = min(w + 4 * i, NR - 1);
    v[i] = s_acc[0][j][lane] + s_acc[1][j][lane] + s_acc[2][j][lane] + s_acc[3][j][lane];
  }
}

// Few rows: t [split][m][16 NR] of the K range of split blockIdx.y for the
// group that begins at row blockIdx.x.
template <int NR>
__global__ __launch_bounds__(256) void lora_shrink_kernel(Lora p) {
  constexpr int RP = 16 * NR;
  __shared__ int s_rows[16];
  __shared__ f32x4 s_acc[4][NR][64];
  const int r = blockIdx.x, a = __builtin_amdgcn_readfirstlane(p.adapter[r]);
  if (!has_adapter(p, a)) return;
  const int n = __builtin_amdgcn_readfirstlane(gather_group(p, r, a, s_rows));
  if (n == 0) return;
  __syncthreads();
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, lg = lane >> 4, rank = rank_of(p, a);
  const int steps = (p.k + 31) / 32, ns = gridDim.y;
  const int s0 = (int)((int64_t)blockIdx.y * steps / ns), s1 = (int)((int64_t)(blockIdx.y + 1) * steps / ns);
  f32x4 v[(NR + 3) / 4];
  shrink_group<NR>(p, a, rank, n, s_rows, s0, s1, s_acc, v);
  float* t = p.t + (int64_t)blockIdx.y * p.m * RP;
#pragma unroll
  for (int i = 0; i < (NR + 3) / 4; ++i) {
    const int k = (w + 4 * i) * 16 + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (k < RP && lg * 4 + e < n) t[(int64_t)s_rows[lg * 4 + e] * RP + k] = k < rank ? v[i][e] : 0.f;
  }
}

// Many rows: the same for a tile's rows.  x and A go through LDS, 64 of k at a
// time, as whole 128-byte lines that are read once per workgroup (with
// fragments straight from memory, 16 rows of 64 bytes an instruction, and each
// wave's own copy of A, 4099 rows of 4096 by 64 ranks took 24.7 us, so 15.4,
// and 18.5 with plan_tile); two tiles of k are in flight while one is
// multiplied.  Wave w has rows 16 w .. 16 w + 15.  The workgroups of a K range
// meet on one XCD where there are a multiple of eight ranges, so that each L2
// holds its share of A.
template <int NR>
__global__ __launch_bounds__(256) void lora_shrink_tile_kernel(Lora p) {
  constexpr int RP = 16 * NR, KT = 64, PITCH = KT + 8, DEPTH = 2;
  constexpr int NXL = kTile * 8 / 256, NAL = (RP * 8 + 255) / 256;   // 16-byte pieces a thread
  union Lds {
    PlanLds plan;
    struct {
      _Float16 x[2][kTile][PITCH], a[2][RP][PITCH];
    } stage;
  };
  __shared__ __attribute__((aligned(16))) Lds s_lds;
  auto &s_x = s_lds.stage.x;
  auto &s_a = s_lds.stage.a;
  __shared__ int s_rows[kTile];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, lg = lane >> 4;
  int a;
  const int n = plan_tile(p, blockIdx.y, s_lds.plan, s_rows, a);
  if (blockIdx.x == 0) {                 // the tile, for the second product
    if (tid == 0) p.tile_adapter[blockIdx.y] = n ? a : -1;
    if (tid < kTile) p.tile_rows[blockIdx.y * kTile + tid] = tid < n ? s_rows[tid] : -1;
  }
  if (n == 0 || a == p.n_adapters) return;
  const int tiles = (p.k + KT - 1) / KT, ns = gridDim.x;
  const int t0 = (int)((int64_t)blockIdx.x * tiles / ns), nt = (int)((int64_t)(blockIdx.x + 1) * tiles / ns) - t0;
  float* t = p.t + (int64_t)blockIdx.x * p.m * RP;
  const int rank = rank_of(p, a);
  const int seg = (tid & 7) * 8;
  const _Float16 *xp[NXL], *ap[NAL];
#pragma unroll
  for (int e = 0; e < NXL; ++e) xp[e] = p.x + (int64_t)s_rows[min((tid >> 3) + 32 * e, n - 1)] * p.k + seg;
#pragma unroll
  for (int e = 0; e < NAL; ++e)
    ap[e] = p.a + ((int64_t)a * p.R + max(min((tid >> 3) + 32 * e, rank - 1), 0)) * p.k + seg;
  f16x8 xr[DEPTH][NXL], ar[DEPTH][NAL];
  auto load = [&](int i, int tile) {
    const int k = (t0 + tile) * KT;
    const bool in = k + seg < p.k;         // k is a multiple of 8
#pragma unroll
    for (int e = 0; e < NXL; ++e) {
      xr[i][e] = *reinterpret_cast<const f16x8*>(xp[e] + (in ? k : -seg));
      if (!in) xr[i][e] = f16x8{};
    }
#pragma unroll
    for (int e = 0; e < NAL; ++e) {
      ar[i][e] = *reinterpret_cast<const f16x8*>(ap[e] + (in ? k : -seg));
      if (!in) ar[i][e] = f16x8{};
    }
  };
  f32x4 acc[NR];
#pragma unroll
  for (int j = 0; j < NR; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // one tile of k: its loads' registers take those of the tile DEPTH later
  auto step = [&](int i, int tile, bool more) {
    const int buf = tile & 1;
#pragma unroll
    for (int e = 0; e < NXL; ++e) *reinterpret_cast<f16x8*>(&s_x[buf][(tid >> 3) + 32 * e][seg]) = xr[i][e];
#pragma unroll
    for (int e = 0; e < NAL; ++e)
      if ((tid >> 3) + 32 * e < RP) *reinterpret_cast<f16x8*>(&s_a[buf][(tid >> 3) + 32 * e][seg]) = ar[i][e];
    if (more) load(i, tile + DEPTH);
    __syncthreads();     // the buffer before last was read before the previous tile's barrier
#pragma unroll
    for (int ks = 0; ks < KT / 32; ++ks) {
      const f16x8 xv = *reinterpret_cast<const f16x8*>(&s_x[buf][w * 16 + col][ks * 32 + lg * 8]);
#pragma unroll
      for (int j = 0; j < NR; ++j) {
        if (j * 16 >= rank) break;
        const f16x8 av = *reinterpret_cast<const f16x8*>(&s_a[buf][j * 16 + col][ks * 32 + lg * 8]);
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv, av, acc[j], 0, 0, 0);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < DEPTH; ++i) load(i, min(i, nt - 1));
  int tb = 0;
  for (; tb + 2 * DEPTH <= nt; tb += DEPTH) {
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) step(i, tb + i, true);
  }
#pragma unroll
  for (int i = 0; i < 2 * DEPTH - 1; ++i)
    if (tb + i < nt) step(i % DEPTH, tb + i, tb + i + DEPTH < nt);
#pragma unroll
  for (int j = 0; j < NR; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = w * 16 + lg * 4 + e;
      if (at < n) t[(int64_t)s_rows[at] * RP + j * 16 + col] = j * 16 + col < rank ? acc[j][e] : 0.f;
    }
}

// Ranks j .. j + 3 of row r's t: the splits added in order.
template <int NR>
__device__ __forceinline__ f32x4 t_sum(const Lora& p, int r, int j) {
  const float* t = p.t + (int64_t)r * (16 * NR) + j;
  f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < p.n_split; ++s) v += *reinterpret_cast<const f32x4*>(t + (int64_t)s * p.m * (16 * NR));
  return v;
}

__device__ __forceinline__ float scale_of(const Lora& p, int a) { return p.scale ? p.scale[a] : 1.f; }

// The upper 16 bits of two fp32 values as two bf16, and what is left of a value
// without them.
__device__ __forceinline__ uint32_t tops(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
}
__device__ __forceinline__ float rest(float v) { return v - __uint_as_float(__float_as_uint(v) & 0xffff0000u); }

// t of a group's 16 rows in LDS, in three bf16 parts that add up to it.  Only
// the first part of an infinite or NaN value means something.
template <int NR>
struct GroupParts {
  static constexpr int RP = 16 * NR, KS = (RP + 31) / 32, PITCH = KS * 32 + 8;
  uint16_t part[3][16][PITCH];

  // ranks j .. j + 3 of row i
  __device__ __forceinline__ void put(int i, int j, f32x4 v) {
#pragma unroll
    for (int c = 0; c < 3; ++c) {
      *reinterpret_cast<uint2*>(&part[c][i][j]) = make_uint2(tops(v[0], v[1]), tops(v[2], v[3]));
      if (RP < KS * 32) *reinterpret_cast<uint2*>(&part[c][i][RP + j]) = make_uint2(0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = rest(v[e]);
    }
  }
  // row col's ranks of K step j
  __device__ __forceinline__ bf16x8 get(int c, int col, int j) const {
    return *reinterpret_cast<const bf16x8*>(&part[c][col][j * 32 + ((threadIdx.x & 63) >> 4) * 8]);
  }
};

// Eight f16 values of B in two bf16 parts that add up to them (of an infinite or
// NaN one the first alone).
__device__ __forceinline__ void split_b(f16x8 b, bf16x8& hi, bf16x8& lo) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  u32x4 h, l;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = (float)b[2 * e], y = (float)b[2 * e + 1];
    h[e] = tops(x, y);
    l[e] = tops(rest(x), rest(y));
  }
  hi = __builtin_bit_cast(bf16x8, h);
  lo = __builtin_bit_cast(bf16x8, l);
}

// y += scale t B^T for NX groups of 16 rows and 16 CT columns.  The first parts'
// product is summed apart from the others': where t or B are infinite or NaN it
// is what the sum is, and the others mean nothing.  Columns of two groups come
// one after the other, which leaves registers to a fourth wave a SIMD (4099 rows
// of rank 64: 54.8 us, two columns at a time 57.8); those of one all together.
template <int NR, int NX, int CT>
__device__ __forceinline__ void expand_columns(const GroupParts<NR> (&t)[NX], int rank, float scale,
                                               const f16x8 (&b)[GroupParts<NR>::KS][CT], f32x4 (&y)[NX][CT]) {
  constexpr int CG = NX == 1 ? CT : 1;
  const int col = threadIdx.x & 15;
#pragma unroll
  for (int c0 = 0; c0 < CT; c0 += CG) {
    f32x4 d[CG][NX], d_lo[CG][NX];
#pragma unroll
    for (int c = 0; c < CG; ++c)
#pragma unroll
      for (int i = 0; i < NX; ++i) d[c][i] = d_lo[c][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < GroupParts<NR>::KS; ++j) {
      if (j * 32 >= rank) break;
      bf16x8 hi[CG], lo[CG];
#pragma unroll
      for (int c = 0; c < CG; ++c) split_b(b[j][c0 + c], hi[c], lo[c]);
#pragma unroll
      for (int part = 2; part >= 0; --part) {
#pragma unroll
        for (int i = 0; i < NX; ++i) {
          const bf16x8 tp = t[i].get(part, col, j);
#pragma unroll
          for (int c = 0; c < CG; ++c) {
            d_lo[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo[c], tp, d_lo[c][i], 0, 0, 0);
            f32x4& sum = part ? d_lo[c][i] : d[c][i];
            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi[c], tp, sum, 0, 0, 0);
          }
        }
      }
    }
#pragma unroll
    for (int c = 0; c < CG; ++c)
#pragma unroll
      for (int i = 0; i < NX; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = d[c][i][e];
          y[i][c0 + c][e] = __builtin_fmaf(fabsf(v) < INFINITY ? v + d_lo[c][i][e] : v, scale, y[i][c0 + c][e]);
        }
  }
}

// B of columns c0 + 16 c + l % 16, ranks 32 j + 8 (l / 16) .. + 7; ranks that
// do not count are zero (the last eight that exist are read there).
template <int KS, int CT>
__device__ __forceinline__ void load_b(const Lora& p, int a, int rank, int c0, f16x8 (&b)[KS][CT]) {
  const int lane = threadIdx.x & 63, col = lane & 15, lg = lane >> 4;
#pragma unroll
  for (int j = 0; j < KS; ++j)
#pragma unroll
    for (int c = 0; c < CT; ++c)
      b[j][c] = *reinterpret_cast<const f16x8*>(p.b + ((int64_t)a * p.n + min(c0 + c * 16 + col, p.n - 1)) * p.R +
                                                min(j * 32 + lg * 8, max(rank - 1, 0) & ~7));
#pragma unroll
  for (int j = 0; j < KS; ++j)
    if (j * 32 + 32 > rank) {
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) b[j][c][e] = j * 32 + lg * 8 + e < rank ? b[j][c][e] : (_Float16)0.f;
    }
}

// The base's values of one row at columns c0 + 16 c + 4 lg .. + 3, and y's.
// Columns past n take the last one's: with a zero for each under a condition, the
// wide second product of rank 64 kept 16 bytes a thread in scratch (4099 rows 62.9
// for 60.1 us).
template <int CT>
__device__ __forceinline__ void load_base(const Lora& p, int row, int c0, int lg, bool whole, f32x4 (&y)[CT]) {
  const float* b = p.base + (int64_t)row * p.y_stride;
  if (whole) {
#pragma unroll
    for (int c = 0; c < CT; ++c) y[c] = *reinterpret_cast<const f32x4*>(b + c0 + c * 16 + lg * 4);
  } else {
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int at = c0 + c * 16 + lg * 4 + e;
        y[c][e] = b[min(at, p.n - 1)];
      }
  }
}
template <int CT>
__device__ __forceinline__ void store_y(const Lora& p, int row, int c0, int lg, bool whole, const f32x4 (&y)[CT]) {
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int at = c0 + c * 16 + lg * 4;
    float* o = p.y + (int64_t)row * p.y_stride + at;
    if (whole) {
      *reinterpret_cast<f32x4*>(o) = y[c];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (at + e < p.n) o[e] = y[c][e];
    }
  }
}

template <int NR, int CT>
__device__ __forceinline__ void expand_group(const Lora& p, int a, int rank, int n, const int* s_rows,
                                             const GroupParts<NR> (&t)[1], int c0, f32x4 (&y)[1][CT]) {
  constexpr int KS = GroupParts<NR>::KS;
  const int lane = threadIdx.x & 63, col = lane & 15, lg = lane >> 4;
  const float scale = scale_of(p, a);
  f16x8 b[KS][CT];
  load_b<KS, CT>(p, a, rank, c0, b);
  expand_columns<NR, 1, CT>(t, rank, scale, b, y);
  if (col >= n) return;
  store_y<CT>(p, s_rows[col], c0, lg, c0 + 16 * CT <= p.n, y[0]);
}

// A row without an adapter is the base's: columns c0 .. c0 + cols - 1.
__device__ __forceinline__ void copy_row(const Lora& p, int r, int c0, int cols) {
  const int c = c0 + threadIdx.x;
  if (p.y != p.base && (int)threadIdx.x < cols && c < p.n) p.y[r * p.y_stride + c] = p.base[r * p.y_stride + c];
}

// Few rows, second product: the group that begins at row `block`, 256 columns.
// Workgroup b runs on XCD b % 8: it serves every eighth row block, whose
// column ranges follow each other, so that t is read into one L2 and the rows
// in flight cover whole lines of all memory channels.
template <int NR>
__global__ __launch_bounds__(256) void lora_expand_kernel(Lora p) {
  __shared__ int s_rows[16];
  __shared__ __attribute__((aligned(16))) GroupParts<NR> s_t[1];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cols = (p.n + kColsWg - 1) / kColsWg, rest = blockIdx.x >> 3;
  const int r = rest / cols * 8 + (blockIdx.x & 7), c_wg = rest % cols * kColsWg, c0 = c_wg + w * 64;
  if (r >= p.m) return;
  const int a = __builtin_amdgcn_readfirstlane(p.adapter[r]);
  if (!has_adapter(p, a)) {
    copy_row(p, r, c_wg, kColsWg);
    return;
  }
  const int n = __builtin_amdgcn_readfirstlane(gather_group(p, r, a, s_rows));
  if (n == 0) return;
  __syncthreads();
  f32x4 y[1][4];                           // goes out first, needed last
  load_base<4>(p, s_rows[min(lane & 15, n - 1)], c0, lane >> 4, c0 + 64 <= p.n, y[0]);
  for (int idx = threadIdx.x; idx < n * 4 * NR; idx += 256) {
    const int i = idx / (4 * NR), j = idx % (4 * NR) * 4;
    s_t[0].put(i, j, t_sum<NR>(p, s_rows[i], j));
  }
  __syncthreads();
  if (c0 < p.n) expand_group<NR, 4>(p, a, rank_of(p, a), n, s_rows, s_t, c0, y);
}

// Very few rows: both products in one launch.  Every workgroup of a group's
// column ranges forms t for itself, reading A again (from the L2): dearer
// than a second launch where A is long or the ranges are many (lora_fused).
template <int NR>
__global__ __launch_bounds__(256) void lora_fused_kernel(Lora p) {
  constexpr int RP = 16 * NR, CT = kColsFused / 64;
  __shared__ int s_rows[16];
  __shared__ f32x4 s_acc[4][NR][64];
  __shared__ float s_sum[16][RP + 4];
  __shared__ __attribute__((aligned(16))) GroupParts<NR> s_t[1];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, lg = lane >> 4;
  const int r = blockIdx.y, c_wg = blockIdx.x * kColsFused, c0 = c_wg + w * 16 * CT;
  const int a = __builtin_amdgcn_readfirstlane(p.adapter[r]);
  if (!has_adapter(p, a)) {
    copy_row(p, r, c_wg, kColsFused);
    return;
  }
  const int n = __builtin_amdgcn_readfirstlane(gather_group(p, r, a, s_rows));
  if (n == 0) return;
  __syncthreads();
  f32x4 y[1][CT];
  load_base<CT>(p, s_rows[min(col, n - 1)], c0, lg, c0 + 16 * CT <= p.n, y[0]);
  const int rank = rank_of(p, a);
  f32x4 v[(NR + 3) / 4];
  shrink_group<NR>(p, a, rank, n, s_rows, 0, (p.k + 31) / 32, s_acc, v);
#pragma unroll
  for (int i = 0; i < (NR + 3) / 4; ++i) {
    const int k = (w + 4 * i) * 16 + col;
    if (k < RP) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s_sum[lg * 4 + e][k] = k < rank ? v[i][e] : 0.f;
    }
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < n * 4 * NR; idx += 256) {
    const int i = idx / (4 * NR), j = idx % (4 * NR) * 4;
    s_t[0].put(i, j, f32x4{s_sum[i][j], s_sum[i][j + 1], s_sum[i][j + 2], s_sum[i][j + 3]});
  }
  __syncthreads();
  if (c0 < p.n) expand_group<NR, CT>(p, a, rank, n, s_rows, s_t, c0, y);
}

// Many rows, second product: half a tile's rows x COLS columns, 64 a wave; the
// workgroup adds the splits of its rows' t itself (a launch between the two
// that prepared t once cost 1.5-4 us more, whatever the rows).  Workgroups are
// numbered as above.  4099 rows of 4096 columns, rank 64: 43.7 us, where rows
// without an adapter (base to y alone, in this order) take 29.2; the rest is t
// and B, which every half tile reads from the L2.  100 MB come from memory, where
// base, t and B once each are 79: B enters each of the eight L2s.  A whole tile a
// workgroup is as fast, a quarter slower by a seventh; the base's loads ahead of
// the others' slower.  Wide ranges of rank 64 at four waves a SIMD against three:
// 60.3 and 63.8 us for both launches; with 512 rows, which do not fill the chip,
// four were slower (20.2 for 19.3) in ranges of 256.
template <int NR, int COLS>
__global__ __launch_bounds__(COLS, NR == 4 && COLS == 512 ? 4 : 1) void lora_expand_tile_kernel(Lora p) {
  constexpr int KS = GroupParts<NR>::KS, ROWS = kTile / 2, NX = ROWS / 16, PER = (ROWS * 4 * NR + COLS - 1) / COLS;
  __shared__ __attribute__((aligned(16))) GroupParts<NR> s_t[NX];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, lg = lane >> 4;
  const int cols = (p.n + COLS - 1) / COLS, rest = blockIdx.x >> 3;
  const int block = rest / cols * 8 + (blockIdx.x & 7), c0 = rest % cols * COLS + w * 64;
  if (block >= 2 * p.tiles) return;
  const int a = __builtin_amdgcn_readfirstlane(p.tile_adapter[block / 2]);
  const bool with = has_adapter(p, a);
  if (a < 0 || (!with && p.y == p.base)) return;
  const int32_t* list = p.tile_rows + block * ROWS;
  const int first = __builtin_amdgcn_readfirstlane(list[0]);
  if (first < 0) return;                   // a tile's rows fill it from the front
  int rows[NX];
  bool in[NX];
#pragma unroll
  for (int i = 0; i < NX; ++i) {
    rows[i] = list[i * 16 + col];
    in[i] = rows[i] >= 0;
    if (!in[i]) rows[i] = first;           // loads of a row that exists stand in
  }
  const bool whole = c0 + 64 <= p.n;       // no column of the wave lies past n
  f32x4 y[NX][4];
  if (with) {
    f32x4 t[PER];
    int at[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int r = list[min((int)(threadIdx.x + COLS * e) / (4 * NR), ROWS - 1)];
      at[e] = r < 0 ? first : r;
      t[e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    constexpr int FLIGHT = NR <= 4 ? 8 : 4;      // as many loads in flight as registers hold
#pragma unroll FLIGHT
    for (int s = 0; s < p.n_split; ++s)
#pragma unroll
      for (int e = 0; e < PER; ++e)
        t[e] += *reinterpret_cast<const f32x4*>(p.t + ((int64_t)s * p.m + at[e]) * (16 * NR) + threadIdx.x % (4 * NR) * 4);
    const float scale = scale_of(p, a);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = (threadIdx.x + COLS * e) / (4 * NR);
      if (i < ROWS) s_t[i / 16].put(i % 16, threadIdx.x % (4 * NR) * 4, t[e]);
    }
    __syncthreads();
    if (c0 >= p.n) return;
    const int rank = rank_of(p, a);
    f16x8 b[KS][4];
    load_b<KS, 4>(p, a, rank, c0, b);
#pragma unroll
    for (int i = 0; i < NX; ++i) load_base<4>(p, rows[i], c0, lg, whole, y[i]);
    expand_columns<NR, NX, 4>(s_t, rank, scale, b, y);
  } else {
    if (c0 >= p.n) return;
#pragma unroll
    for (int i = 0; i < NX; ++i) load_base<4>(p, rows[i], c0, lg, whole, y[i]);
  }
#pragma unroll
  for (int i = 0; i < NX; ++i)
    if (in[i]) store_y<4>(p, rows[i], c0, lg, whole, y[i]);
}

int rank_tiles(int R) { return R <= 16 ? 1 : R <= 32 ? 2 : R <= 64 ? 4 : 8; }

// Both products in one launch: where a workgroup's A is at most 64 KB and all
// that the workgroups read of it at most 16 MB.  Measured in a graph, one
// launch against two: 2048 x 2048, rank 16 (64 KB), 1 row 6.1 against 7.2 us,
// 16 rows with an adapter each (16 MB) 6.3 against 7.4, 32 rows 8.6 against
// 7.3; 4096 x 4096, rank 16 (128 KB), 1 row 8.2 against 7.2; 256 x 1024 (8 KB),
// 32 rows 4.3 against 7.2.
bool lora_fused(const Lora& p) {
  const int64_t a_bytes = (int64_t)p.R * p.k * 2, ranges = (p.n + kColsFused - 1) / kColsFused;
  return p.m <= kGatherRows && a_bytes <= (64 << 10) && a_bytes * ranges * p.m <= (16 << 20);
}

// The second product of many rows in ranges of 512 columns: halves what its
// workgroups read of t, where ranks are many and the workgroups still fill the
// chip.  512 against 256, both launches, 4096 x 4096, 4 adapters: rank 64, 4096
// rows 45.5 against 48.4 us, 1024 (512 workgroups of 256) 22.5 against 24.0, 512
// rows 18.9 against 17.5; rank 128, 4096 rows 68.6 against 75.3, 512 26.0 against
// 24.4; rank 16, 4096 rows, with f16 halves of t 42.2 against 42.0.
bool lora_wide(const Lora& p) { return (int64_t)(p.m + kTile / 2 - 1) / (kTile / 2) * ((p.n + 255) / 256) >= 512; }

template <int NR>
void launch_lora_nr(const Lora& p, hipStream_t s) {
  auto grid = [&](int blocks, int cols) { return dim3((unsigned)((blocks + 7) / 8 * 8 * ((p.n + cols - 1) / cols))); };
  if (lora_fused(p)) {
    hipLaunchKernelGGL(lora_fused_kernel<NR>, dim3((p.n + kColsFused - 1) / kColsFused, p.m), dim3(256), 0, s, p);
  } else if (p.m <= kGatherRows) {
    hipLaunchKernelGGL(lora_shrink_kernel<NR>, dim3(p.m, p.n_split), dim3(256), 0, s, p);
    hipLaunchKernelGGL(lora_expand_kernel<NR>, grid(p.m, kColsWg), dim3(256), 0, s, p);
  } else {
    hipLaunchKernelGGL(lora_shrink_tile_kernel<NR>, dim3(p.n_split, p.tiles), dim3(256), 0, s, p);
    if constexpr (NR >= 4) {
      if (lora_wide(p)) {
        hipLaunchKernelGGL((lora_expand_tile_kernel<NR, 512>), grid(2 * p.tiles, 512), dim3(512), 0, s, p);
        return;
      }
    }
    hipLaunchKernelGGL((lora_expand_tile_kernel<NR, 256>), grid(2 * p.tiles, 256), dim3(256), 0, s, p);
  }
}

// Tiles that rows of at most so many adapters (and of none) can make.
int most_tiles(int m, int n_adapters) {
  const int sorted = m / kTile + (n_adapters + 1 < m ? n_adapters + 1 : m), runs = most_runs(m);
  return sorted > runs ? sorted : runs;
}

// K splits: enough workgroups for the chip, at least two steps of 32 a wave, at
// most 16 (few rows) or 32.  With at most 8, 1 row of 8960 x 1536, rank 64,
// takes 11.5 for 9.8 us, 512 rows of 14336 x 4096, rank 16, 21.1, with 16 17.3,
// with 32 16.2; 33 rows of the latter with 32 12.9 for 11.6.  Half the
// workgroups for many rows: 4096 of the latter 55.2 for 49.0 us; twice: 50.6.
constexpr int kFewBlocks = 1024, kManyBlocks = 520;

int most_splits(int m, int k) {
  const int most = (k + 31) / 32 / 8, cap = m <= kGatherRows ? 16 : 32;
  return most < 1 ? 1 : most > cap ? cap : most;
}

int lora_splits(int m, int k) {
  const int groups = m <= kGatherRows ? m : (m - 1) / kTile + 1;
  const int want = (m <= kGatherRows ? kFewBlocks : kManyBlocks) / groups, most = most_splits(m, k);
  return want < 1 ? 1 : want > most ? most : want;
}

// The workspace of a call of up to m <= kPlanRows rows: every part grows with
// m, so that one for the largest call serves all.
struct LoraWs {
  int64_t t, tile_adapter, tile_rows, bytes;
};
LoraWs lora_ws(int m, int k, int R, int n_adapters) {
  LoraWs w{};
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += (bytes + 15) / 16 * 16;
    return here;
  };
  const int64_t rp = rank_tiles(R) * 16;
  // splits x rows of t: at most the workgroups wanted times a group's rows
  const int64_t most = m <= kGatherRows ? kFewBlocks : kManyBlocks * kTile, all = (int64_t)most_splits(m, k) * m;
  w.t = take((all < most ? all : most) * rp * 4);
  if (m > kGatherRows) {
    w.tile_adapter = take((int64_t)most_tiles(m, n_adapters) * 4);
    w.tile_rows = take((int64_t)most_tiles(m, n_adapters) * kTile * 4);
  }
  w.bytes = at;
  return w;
}

}  // namespace

bool lora_fits(int m, int n, int n_adapters) {
  const int rows = m < kPlanRows ? m : kPlanRows;
  const int64_t blocks = rows <= kGatherRows ? rows : 2 * most_tiles(rows, n_adapters);
  return (blocks + 7) / 8 * 8 * ((n - 1) / 512 + 1) * 2 <= kMaxBlocks;      // in 256 threads
}

int64_t lora_ws_bytes(int m, int k, int R, int n_adapters) {
  return lora_ws(m < kPlanRows ? m : kPlanRows, k, R, n_adapters).bytes;
}

void launch_lora(Lora p, void* ws, hipStream_t s) {
  const int rows = p.m;
  for (int64_t r = 0; r < rows; r += kPlanRows) {
    Lora q = p;
    q.m = rows - r < kPlanRows ? (int)(rows - r) : kPlanRows;
    q.x += r * q.k;
    q.adapter += r;
    q.base += r * q.y_stride;
    q.y += r * q.y_stride;
    const LoraWs w = lora_ws(q.m, q.k, q.R, q.n_adapters);
    uint8_t* b = reinterpret_cast<uint8_t*>(ws);
    q.t = reinterpret_cast<float*>(b + w.t);
    q.tile_adapter = reinterpret_cast<int32_t*>(b + w.tile_adapter);
    q.tile_rows = reinterpret_cast<int32_t*>(b + w.tile_rows);
    q.tiles = most_tiles(q.m, q.n_adapters);
    q.n_split = lora_splits(q.m, q.k);
    switch (rank_tiles(q.R)) {
      case 1: launch_lora_nr<1>(q, s); break;
      case 2: launch_lora_nr<2>(q, s); break;
      case 4: launch_lora_nr<4>(q, s); break;
      default: launch_lora_nr<8>(q, s); break;
    }
  }
}

}  // namespace mzk
