// Attention of several new tokens of every sequence of a batch, trees or
// chains, over its chunked KV cache (gfx950): for node i of sequence b, head h
// of KV head h / G,
//   out = sum_j w_j v_j / sum_j w_j,  w_j = 2^(s_j - max s),
//   s_j = log2(e) / sqrt(hd) q . k_j,  j < len or j = len + t, t in the node's mask.
//
// The G T query heads and nodes of a KV head are the columns of the products,
// R at a time, so that a key is read once for R of them.  As in
// attention_batch.hip the work is cut by keys, not by sequences: the units of 64
// or 128 keys of all (sequence, KV head, R columns) lie in one line, each
// workgroup takes an even share of it, and a second kernel joins what several
// shares summed, in a fixed order.
//
// P goes into the products as two f16 values, hi + lo, of 2^(bias + s - max): 22
// bits of a weight (and what it holds down to 2^-34 of the largest), so that an
// output's only rounding to fewer bits is its own.  Both enter the same fp32
// sums.  A weight of 0 removes what a node does not see, unless the value is
// infinite or NaN: then sums that are not finite show it, and the second
// kernel takes the columns that they belong to again, a (row, head) at a time, with
// fp32 products of what the row sees alone.
#include <algorithm>

#include "mz_kernels.h"

namespace mzk {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

struct Seq {
  int first, nodes, len, keys;      // rows first .. first + nodes - 1, keys before the tree and in all
  int tiles, units;                 // of R columns, of UNIT keys
};
template <int R, int UNIT>
__device__ __forceinline__ Seq seq_of(const AttnTree& a, int b) {
  Seq s;
  s.first = min(max(a.row_off[b], 0), a.m);
  s.nodes = min(max(a.row_off[b + 1], s.first), a.m) - s.first;
  if (a.mask) s.nodes = min(s.nodes, 32 * a.mask_words);
  const int top = a.n_table << a.cshift;
  s.len = min(max(a.lens[b], 0), top);
  s.keys = s.nodes < top - s.len ? s.len + s.nodes : top;
  s.tiles = (s.nodes * a.group + R - 1) / R;
  s.units = (s.keys + UNIT - 1) / UNIT;
  return s;
}

__device__ __forceinline__ int shares(const AttnTree& a, int total) { return min(a.wgs, total); }

// The workgroup whose share [g total / nw, (g + 1) total / nw) holds unit u.
__device__ __forceinline__ int share_of(int u, int nw, int total) {
  return (int)((((uint64_t)u + 1) * nw - 1) / (unsigned)total);
}

// Inclusive sum over the 64 NW threads; sum: of all.
template <int NW>
__device__ __forceinline__ int block_scan(int v, int* red, int& sum) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();
  if (lane == 63) red[w] = v;
  __syncthreads();
  int before = 0;
  sum = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    if (i < w) before += red[i];
    sum += red[i];
  }
  return v + before;
}

// A workgroup's share [u, end) of the units, and the sequence that it begins
// in, whose units begin at `first`.  The second kernel's tables on the way: the
// units before every sequence, and the sequence of every row.
struct Share {
  int u, end, b, first;
};
template <int R, int UNIT, int NW>
__device__ __forceinline__ bool share_begin(const AttnTree& a, int* s_red, int* s_at, Share& sh) {
  constexpr int NT = 64 * NW;
  for (int b = blockIdx.x; b <= a.n_seq; b += gridDim.x) {
    if (b < a.n_seq) {
      const Seq s = seq_of<R, UNIT>(a, b);
      const int end = min(max(a.row_off[b + 1], s.first), a.m);
      for (int r = s.first + threadIdx.x; r < end; r += NT) a.row_seq[r] = r - s.first < s.nodes ? b : -1;
    } else {
      const int before = min(max(a.row_off[0], 0), a.m), last = min(max(a.row_off[a.n_seq], before), a.m);
      for (int i = threadIdx.x; i < before + a.m - last; i += NT) a.row_seq[i < before ? i : last + i - before] = -1;
    }
  }
  int total = 0, u_mine = 0, u_before = 0;
  auto units = [&](int b) {
    if (b >= a.n_seq) return 0;
    const Seq s = seq_of<R, UNIT>(a, b);
    return s.tiles * s.units;
  };
  for (int b0 = 0; b0 < a.n_seq; b0 += NT) {
    const int b = b0 + threadIdx.x;
    u_mine = units(b);
    int sum;
    u_before = total + block_scan<NW>(u_mine, s_red, sum) - u_mine;
    if (blockIdx.x == 0 && b < a.n_seq) a.base[b] = u_before;
    total += sum;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.base[a.n_seq] = total;
  const int n_units = total * a.nkv, nw = shares(a, n_units), g = blockIdx.x;
  if (g >= nw) return false;
  sh.u = (int)((uint64_t)g * n_units / nw);
  sh.end = (int)(((uint64_t)g + 1) * n_units / nw);
  auto here = [&](int b) {
    if (sh.u >= u_before * a.nkv && sh.u < (u_before + u_mine) * a.nkv) {
      s_at[0] = b;
      s_at[1] = u_before;
    }
  };
  if (a.n_seq > NT) {
    int run = 0;
    for (int b0 = 0; b0 < a.n_seq; b0 += NT) {
      u_mine = units(b0 + threadIdx.x);
      int sum;
      u_before = run + block_scan<NW>(u_mine, s_red, sum) - u_mine;
      here(b0 + threadIdx.x);
      run += sum;
    }
  } else {
    here(threadIdx.x);
  }
  __syncthreads();
  sh.b = __builtin_amdgcn_readfirstlane(s_at[0]);
  sh.first = __builtin_amdgcn_readfirstlane(s_at[1]) * a.nkv;
  return true;
}

// The share's next piece: units t0 .. t1 - 1 of columns tile R .. of KV head h of sequence s.
struct Piece {
  int h, tile, t0, t1;
};
template <int R, int UNIT>
__device__ __forceinline__ Piece next_piece(const AttnTree& a, Share& sh, Seq& s) {
  if (sh.u >= sh.first + s.tiles * s.units * a.nkv) {      // past this sequence: on to the next that has rows, 64 in a look
    const int lane = threadIdx.x & 63;
    sh.first += s.tiles * s.units * a.nkv;
    uint64_t some = 0;
    for (++sh.b; !some; sh.b += some ? __builtin_ctzll(some) : 64)
      some = __ballot(sh.b + lane >= a.n_seq || seq_of<R, UNIT>(a, sh.b + lane).nodes > 0);
    s = seq_of<R, UNIT>(a, sh.b);
  }
  const int pair = (sh.u - sh.first) / s.units, t0 = sh.u - sh.first - pair * s.units, h = pair / s.tiles;
  const Piece p{h, pair - h * s.tiles, t0, min(s.units, t0 + sh.end - sh.u)};
  sh.u += p.t1 - p.t0;
  return p;
}

__device__ __forceinline__ unsigned ones(int n) { return n <= 0 ? 0u : n >= 8 ? 0xFFu : (1u << n) - 1; }
__device__ __forceinline__ uint64_t ones64(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; }

// Whether a node sees key j (before the end); words: its mask.
__device__ __forceinline__ bool sees(const AttnTree& a, const Seq& s, int j, int node, const uint32_t* words) {
  const int at = j - s.len;
  return at < 0 || (a.mask ? (words[at >> 5] >> (at & 31)) & 1 : at <= node);
}

// Which of the eight keys from j on a node sees, of those before the end.
__device__ __forceinline__ unsigned seen8(const AttnTree& a, const Seq& s, int j, int node, const uint32_t* words) {
  const int at = j - s.len;              // of the tree
  unsigned m;
  if (a.mask) {
    if (at <= -8) {
      m = 0xFF;
    } else if (at < 0) {
      m = ones(-at) | (words[0] << -at);
    } else {
      const int w = at >> 5;
      const uint64_t lo = w < a.mask_words ? words[w] : 0, hi = w + 1 < a.mask_words ? words[w + 1] : 0;
      m = (unsigned)((hi << 32 | lo) >> (at & 31));
    }
  } else {
    m = ones(node - at + 1);
  }
  return m & ones(s.keys - j);
}

// The same of 64 keys from j on (the end is not looked at).
__device__ __forceinline__ uint64_t seen64(const AttnTree& a, const Seq& s, int j, int node, const uint32_t* words) {
  const int at = j - s.len;
  if (!a.mask) return ones64(node - at + 1);
  if (at <= -64) return ~0ull;
  auto pair = [&](int w) {               // words w and w + 1
    const uint64_t lo = w < a.mask_words ? words[w] : 0, hi = w + 1 < a.mask_words ? words[w + 1] : 0;
    return hi << 32 | lo;
  };
  if (at < 0) return ones64(-at) | pair(0) << -at;
  const int w = at >> 5, shift = at & 31;
  const uint64_t low = pair(w);
  return shift ? low >> shift | (uint64_t)(w + 2 < a.mask_words ? words[w + 2] : 0) << (64 - shift) : low;
}

// ---- up to 32 columns
// Four waves take the 32-key blocks of a share in turn, each for all R
// columns: S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_16x16x32, K and V^T
// fragments straight from the slots, 16 bytes a lane, since a fragment serves one
// wave only.  Row i of the score product holds key 8 (i / 4) + 4 t + i % 4 of the
// block (t: first or second product), so that the eight scores of a lane are
// eight consecutive keys: its mask is eight bits, and the P operand meets one
// 16-byte run of V^T.  The waves' sums meet in LDS at a piece's end.
constexpr int kFewUnit = 128, kFewWaves = 4, kBlock = 32, kCols = 16, kFewWgs = 512;
constexpr float kFewBias = 14.f;

// Slots of a lane's K rows and of its V^T run in the block at key j0.
struct Slots {
  int k, v;
};
// SMALL: chunks of fewer than 32 tokens, a slot per 8 keys of a lane instead
// of one per block.  (Keys past the last one take its entry.)
template <bool SMALL>
__device__ __forceinline__ Slots slots_of(const int32_t* table, int cshift, int j0, int col, int lg, int last) {
  if constexpr (SMALL) return {table[min(j0 + 8 * (col >> 2), last) >> cshift], table[min(j0 + 8 * lg, last) >> cshift]};
  return {0, table[j0 >> cshift]};
}

template <int HD, int NB, bool SMALL>
__global__ __launch_bounds__(64 * kFewWaves, 2) void tree_few_kernel(AttnTree a) {
  constexpr int R = NB * kCols, UNIT = kFewUnit;
  constexpr int KS = HD / 32;          // 32-wide dimension steps of a score product
  constexpr int DB = HD / 16;          // 16-dimension blocks of the output
  __shared__ float s_o[kFewWaves][DB][4][64];
  __shared__ float s_ml[kFewWaves][2][R];
  __shared__ int s_red[kFewWaves], s_at[2];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, lg = lane >> 4, dkv = a.nkv * HD, g = blockIdx.x;
  Share sh;
  if (!share_begin<R, UNIT, kFewWaves>(a, s_red, s_at, sh)) return;
  Seq s = seq_of<R, UNIT>(a, sh.b);
  while (sh.u < sh.end) {
    const Piece p = next_piece<R, UNIT>(a, sh, s);
    const int32_t* table = a.table + (int64_t)sh.b * a.n_table;
    f16x8 q[NB][KS];
    f32x4 o[NB][DB];
    float m[NB], l[NB];
    int node[NB];
    const uint32_t* words[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int x = p.tile * R + nb * kCols + col, i = x / a.group, head = p.h * a.group + x - i * a.group;
      const bool there = i < s.nodes;
      node[nb] = there ? i : -1;
      words[nb] = a.mask + (int64_t)(s.first + (there ? i : 0)) * a.mask_words;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        q[nb][ks] = f16x8{};
        if (there) q[nb][ks] = *reinterpret_cast<const f16x8*>(a.q + ((int64_t)(s.first + i) * a.nq + head) * HD + ks * 32 + lg * 8);
      }
#pragma unroll
      for (int d = 0; d < DB; ++d) o[nb][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[nb] = -INFINITY;
      l[nb] = 0.f;
    }
    // This wave's blocks: j0, j0 + 128, ... below the piece's end.  Table
    // entries are read a block ahead, so that a block waits for one trip to
    // memory, not two.
    const int j_end = min(p.t1 * UNIT, s.keys), last = s.keys - 1;
    Slots next = slots_of<SMALL>(table, a.cshift, min(p.t0 * UNIT + w * kBlock, last), col, lg, last);
    for (int j0 = p.t0 * UNIT + w * kBlock; j0 < j_end; j0 += UNIT) {
      Slots at = next;
      next = slots_of<SMALL>(table, a.cshift, min(j0 + UNIT, last), col, lg, last);
      const bool ok = (unsigned)at.v < (unsigned)a.n_slots;
      if constexpr (SMALL) {
        if ((unsigned)at.k >= (unsigned)a.n_slots) at.k = 0;
        if (!ok) at.v = 0;
      } else {
        at.k = at.v = __builtin_amdgcn_readfirstlane(at.v);
        if (!ok) continue;
      }
      f16x8 ka[2][KS], va[DB];
      const int kj = j0 + 8 * (col >> 2), vj = j0 + 8 * lg;
      const uint8_t* kp = a.slab + (int64_t)at.k * a.slot_bytes;
      const uint8_t* vp = a.slab + (int64_t)at.v * a.slot_bytes;
      const unsigned k_at = (unsigned)((kj & (a.C - 1)) + (col & 3)) * (unsigned)dkv * 2u + (p.h * HD + lg * 8) * 2u;
      const unsigned v_at = (unsigned)a.C * dkv * 2u + ((unsigned)(p.h * HD + col) * a.C + (vj & (a.C - 1))) * 2u;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          ka[t][ks] = *reinterpret_cast<const f16x8*>(kp + (k_at + (unsigned)(t * 4 * dkv * 2 + ks * 64)));
#pragma unroll
      for (int d = 0; d < DB; ++d)
        va[d] = *reinterpret_cast<const f16x8*>(vp + (v_at + (unsigned)(d * 16 * a.C * 2)));
      const int n_ok = ok ? s.keys - vj : 0;      // keys vj .. vj + n_ok - 1 are there
      const bool tree = j0 + kBlock > s.len;      // part of the block is the tree's, or past it
      if (__any(n_ok < 8)) {                      // values that are not there are not data: zero them
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int i = 0; i < 8; ++i) va[d][i] = i < n_ok ? va[d][i] : (_Float16)0.f;
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        unsigned on = ok && node[nb] >= 0 ? 0xFF : 0;
        if (tree && on) on = seen8(a, s, vj, node[nb], words[nb]);
        f32x4 sc[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ka[t][ks], q[nb][ks], sc[t], 0, 0, 0);
        }
        // A key that counts raises the running max to at least the lowest
        // fp32 value, so -inf means that none was seen; scores of -inf and NaN
        // then go where the formula sends them.
        float e[8], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = sc[i >> 2][i & 3] * a.scale_log2;
          e[i] = (on >> i) & 1 ? v : -INFINITY;
          top = (on >> i) & 1 ? fmaxf(top, fmaxf(v, kLowest)) : top;
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > m[nb])) {
          const float now = fmaxf(m[nb], top);
          const float alpha = now == m[nb] ? 1.f : exp2_hw(m[nb] - now);
          m[nb] = now;
          l[nb] *= alpha;
#pragma unroll
          for (int d = 0; d < DB; ++d) o[nb][d] *= alpha;
        }
        const float base = m[nb] == -INFINITY ? 0.f : m[nb] - kFewBias;
        f16x8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float w8 = exp2_hw(e[i] - base);
          l[nb] += w8;
          hi[i] = (_Float16)w8;
          lo[i] = (_Float16)(w8 - (float)hi[i]);
        }
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          o[nb][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va[d], hi, o[nb][d], 0, 0, 0);
          o[nb][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va[d], lo, o[nb][d], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      l[nb] += __shfl_xor(l[nb], 16);
      l[nb] += __shfl_xor(l[nb], 32);
    }
    __syncthreads();                   // the piece before has been read
    if (lg == 0)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        s_ml[w][0][nb * kCols + col] = m[nb];
        s_ml[w][1][nb * kCols + col] = l[nb];
      }
    // thread: column threadIdx % 16 of a block, output dimensions (threadIdx / 16) DPT .. + DPT
    constexpr int DPT = HD / 16;
    const int c = threadIdx.x & 15, dbase = (threadIdx.x >> 4) * DPT;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (nb) __syncthreads();
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) s_o[w][d][r][lane] = o[nb][d][r];
      __syncthreads();
      const int x = nb * kCols + c, i = (p.tile * R + x) / a.group, head = p.h * a.group + p.tile * R + x - i * a.group;
      float mx = -INFINITY, wt[kFewWaves], den = 0.f;
#pragma unroll
      for (int v = 0; v < kFewWaves; ++v) mx = fmaxf(mx, s_ml[v][0][x]);
#pragma unroll
      for (int v = 0; v < kFewWaves; ++v) {
        const float mv = s_ml[v][0][x];
        wt[v] = mv == -INFINITY ? 0.f : exp2_hw(mv - mx);
        den += wt[v] * s_ml[v][1][x];
      }
      float acc[DPT];
      bool finite = fabsf(den) < INFINITY;
#pragma unroll
      for (int e = 0; e < DPT; ++e) {
        const int dim = dbase + e;
        acc[e] = 0.f;
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v) acc[e] += wt[v] * s_o[v][dim >> 4][dim & 3][((dim >> 2) & 3) * 16 + c];
        finite &= fabsf(acc[e]) < INFINITY;
      }
      const int bad = __syncthreads_or(!finite);
      if (i >= s.nodes) continue;
      const int64_t row = (int64_t)(s.first + i) * a.nq + head;
      if (p.t0 == 0 && p.t1 == s.units) {
        typedef _Float16 out_vec __attribute__((ext_vector_type(DPT)));
        const float inv = mx == -INFINITY ? 0.f : 1.0f / den;
        out_vec y;
#pragma unroll
        for (int e = 0; e < DPT; ++e) y[e] = (_Float16)(acc[e] * inv);
        *reinterpret_cast<out_vec*>(a.out + row * HD + dbase) = y;
        if (dbase == 0) a.again[row] = bad;
      } else {
        const int64_t e0 = (int64_t)(2 * g + (p.t0 == 0)) * R + x;
        if (dbase == 0) a.ml[e0] = make_float2(bad ? NAN : mx, den);
#pragma unroll
        for (int e = 0; e < DPT; e += 4)
          *reinterpret_cast<float4*>(a.part + e0 * HD + dbase + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
      }
    }
  }
}

// ---- more columns
// NW waves own 32 columns each and meet the same keys, 64 at a time, which are
// loaded into LDS once for all of them (global_load_lds, 16 bytes a lane, one
// tile ahead): S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16.  Lane l
// feeds row / column l % 32 with the 8 consecutive k of group l / 32; element r
// of the sums is row 8 (r / 4) + 4 (l / 32) + r % 4.  The score product's row i holds
// the key whose bits 2 and 3 are those of i exchanged, so that a lane's scores are
// eight consecutive keys from 16 g + 8 (l / 32) on, g = 0..3, and the P operand meets
// 16-byte runs of V^T.
//
// A step multiplies: the scores of tile t + 1 while the weights of the first half
// of tile t are formed; then P V of tile t while those of the second half are, and
// the max of tile t + 1.  The running max is raised only where a tile exceeds it
// by more than kSlack, so that sums are seldom scaled.
constexpr int kTile = 64, kWideWaves = 8;      // keys of a tile; waves of a CU, two a SIMD
constexpr float kSlack = 4.f, kWideBias = 11.f;

// LDS tiles are swizzled on 16-byte columns: row r's column c lies at c ^ r % 16
// (K, 256-byte rows), c ^ (r / 2) % 8 (128-byte rows), so that neither the reads
// of 32 rows' same column nor the writes of whole rows meet in a bank.
template <int HALVES>
__device__ __forceinline__ int swizzle(int r, int c) {
  return HALVES == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7);
}
template <int HALVES>
__device__ __forceinline__ int tile_at(int r, int c) { return r * HALVES + swizzle<HALVES>(r, c) * 8; }

template <int HD, int NW, bool SMALL>
__global__ __launch_bounds__(64 * NW, HD == 128 && NW == 2 ? 1 : 2) void tree_wide_kernel(AttnTree a) {
  constexpr int R = 32 * NW, UNIT = kTile;
  constexpr int KC = HD / 8;                                   // 16-byte columns of a key
  constexpr int STRETCHES = kTile * KC / 64;                   // of 1 KB, 64 lanes' 16 bytes, in a tile of K and of V^T
  constexpr int PER = STRETCHES / NW;                          // of a wave
  constexpr int TILE = kTile * HD;                             // halves
  constexpr int KS = HD / 16, TN = HD / 32;
  __shared__ __attribute__((aligned(16))) _Float16 lds[4 * TILE];      // K of two tiles, V^T of two
  __shared__ int s_red[NW], s_at[2];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5, dkv = a.nkv * HD, g = blockIdx.x;
  Share sh;
  if (!share_begin<R, UNIT, NW>(a, s_red, s_at, sh)) return;

  // where the lane's 16 bytes of a stretch come from: stretch i NW + w holds
  // pieces 64 (i NW + w) + lane of the swizzled tile, so that from one i to the next
  // the key (K) or the dimension (V^T) goes on by a multiple of 8, and the column
  // stays as it is but for K of 16 columns and rows that are 8 apart
  constexpr int K_STEP = NW * 64 / KC, V_STEP = NW * 8;
  const int k_row = (w * 64 + lane) / KC, v_row = w * 8 + lane / 8;
  const unsigned k_of = swizzle<HD>(k_row, lane % KC) * 16u;
  const int v_key = swizzle<kTile>(v_row, lane % 8) * 8;       // the first of the eight keys
  static_assert(STRETCHES % NW == 0 && V_STEP % 16 == 0 && K_STEP % 8 == 0, "columns of the stretches");
  typedef __attribute__((address_space(3))) void lds_void;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)lds);
  auto k_buf = [&](int t) { return (t & 1) * TILE; };
  auto v_buf = [&](int t) { return (2 + (t & 1)) * TILE; };
  // 64 lanes' 16 bytes from base + at into LDS.  (The wait state lies between
  // the write of M0 and the load that reads it.)
  auto fetch = [&](const uint8_t* base, unsigned at, int to) {
    const uint32_t m0 = __builtin_amdgcn_readfirstlane(lds0 + to * 2);
    if constexpr (SMALL) {
      const uint8_t* from = base + at;
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(m0), "v"(from) : "memory");
    } else {
      const uint64_t b = (uint64_t)(uintptr_t)base;
      const uint64_t u = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(m0), "v"(at), "s"(u) : "memory");
    }
  };

  Seq s = seq_of<R, UNIT>(a, sh.b);
  while (sh.u < sh.end) {
    const Piece p = next_piece<R, UNIT>(a, sh, s);
    const int32_t* table = a.table + (int64_t)sh.b * a.n_table;
    const int last = s.keys - 1;
    const int x = p.tile * R + w * 32 + col, node = x / a.group, head = p.h * a.group + x - node * a.group;
    const bool there = node < s.nodes;
    const bool active = (p.tile * R + w * 32) / a.group < s.nodes;      // of the wave
    const uint32_t* words = a.mask + (int64_t)(s.first + (there ? node : 0)) * a.mask_words;
    f16x8 q[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      q[ks] = f16x8{};
      if (there) q[ks] = *reinterpret_cast<const f16x8*>(a.q + ((int64_t)(s.first + node) * a.nq + head) * HD + ks * 16 + half * 8);
    }
    f32x16 o[TN];
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
    float m = -INFINITY, l = 0.f;

    // Lane i holds the slot of key i of a tile.
    auto slot_of = [&](int t) { return table[min(t * kTile + lane, last) >> a.cshift]; };
    auto clean = [&](int slot) { return (unsigned)slot < (unsigned)a.n_slots ? slot : 0; };
    auto load_k = [&](int t, int slots) {
      const int at = clean(slots), j0 = (t * kTile) & (a.C - 1);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int row = k_row + i * K_STEP, j = SMALL ? (j0 + row) & (a.C - 1) : j0 + row;
        const int slot = SMALL ? __shfl(at, row) : at;
        const unsigned of = K_STEP % 16 == 0 || KC < 16 ? k_of : k_of ^ (i & 1) * 128u;
        fetch(a.slab + (int64_t)slot * a.slot_bytes, (unsigned)j * (unsigned)dkv * 2u + p.h * HD * 2u + of, k_buf(t) + (i * NW + w) * 512);
      }
    };
    auto load_v = [&](int t, int slots) {
      const int at = clean(slots), j0 = (t * kTile) & (a.C - 1), j = SMALL ? (j0 + v_key) & (a.C - 1) : j0 + v_key;
      const int slot = SMALL ? __shfl(at, v_key) : at;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        fetch(a.slab + (int64_t)slot * a.slot_bytes,
              ((unsigned)(dkv + p.h * HD + v_row + i * V_STEP) * (unsigned)a.C + (unsigned)j) * 2u, v_buf(t) + (i * NW + w) * 512);
    };
    // Keys of tile t that are there, and zeros for the values of the others.
    auto there64 = [&](int t, int slots) { return __ballot((unsigned)slots < (unsigned)a.n_slots && t * kTile + lane < s.keys); };
    auto mend_v = [&](int t, uint64_t keys) {
      const unsigned on = (unsigned)(keys >> v_key) & 0xFF;
      if (on == 0xFF) return;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        f16x8* v = reinterpret_cast<f16x8*>(lds + v_buf(t) + ((i * NW + w) * 64 + lane) * 8);
        f16x8 e = *v;
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = (on >> k) & 1 ? e[k] : (_Float16)0.f;
        *v = e;
      }
    };

    const int krow = (col & ~12) | ((col & 8) >> 1) | ((col & 4) << 1);
    auto k_frag = [&](const _Float16* k, int i) {        // of score product i
      return *reinterpret_cast<const f16x8*>(&k[tile_at<HD>((i & 1) * 32 + krow, (i >> 1) * 2 + half)]);
    };
    auto v_frag = [&](const _Float16* v, int grp, int t) {
      return *reinterpret_cast<const f16x8*>(&v[tile_at<kTile>(t * 32 + col, grp * 2 + half)]);
    };
    // Scores of tile t that do not count become -inf; keys: those that are there.
    auto mask_scores = [&](f32x16 (&sc)[2], int t, uint64_t keys) {
      const uint64_t on = keys & seen64(a, s, t * kTile, node, words);
      const unsigned mine[2] = {(unsigned)(on >> (8 * half)), (unsigned)(on >> (32 + 8 * half))};
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float v = sc[kk][r];
          sc[kk][r] = (mine[kk] >> (16 * (r >> 3) + (r & 7))) & 1 ? v : -INFINITY;
        }
      return on != 0;
    };
    // A tile with a key that counts raises the max to at least the lowest fp32
    // value, so -inf means that none was seen.
    auto raise_max = [&](float mx, bool some) {
      mx = fmaxf(mx, __shfl_xor(mx, 32)) * a.scale_log2;
      if (some) mx = fmaxf(mx, kLowest);
      const bool raise = mx > m + kSlack;
      if (__any(raise)) {
        const float now = raise ? mx : m;
        const float alpha = raise ? exp2_hw(m - now) : 1.f;
        m = now;
        l *= alpha;
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[t][r] *= alpha;
      }
    };
    f16x8 hi[4], lo[4];
    auto weight = [&](const f32x16 (&sc)[2], int i, float base) {      // score i of 32
      const float e = exp2_hw(__builtin_fmaf(sc[i >> 4][i & 15], a.scale_log2, -base));
      l += e;
      const _Float16 h = (_Float16)e;
      hi[i >> 3][i & 7] = h;
      lo[i >> 3][i & 7] = (_Float16)(e - (float)h);
    };

    const int t_end = p.t1;
    int s1 = slot_of(min(p.t0 + 1, t_end - 1)), s2 = slot_of(min(p.t0 + 2, t_end - 1));
    uint64_t keys;
    f32x16 sa[2], sb[2];
    {
      const int s0 = slot_of(p.t0);
      load_k(p.t0, s0);
      load_v(p.t0, s0);
      if (p.t0 + 1 < t_end) load_k(p.t0 + 1, s1);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      keys = there64(p.t0, s0);
      if (~keys) mend_v(p.t0, keys);
      __syncthreads();
      if (active) {
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
          const f32x16 zero = {};
          sa[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k_frag(lds + k_buf(p.t0), i), q[i >> 1], i < 2 ? zero : sa[i & 1], 0, 0, 0);
        }
        bool some = true;
        if (~keys || p.t0 * kTile + kTile > s.len) some = mask_scores(sa, p.t0, keys);
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 32; ++i) mx = fmaxf(mx, sa[i >> 4][i & 15]);
        raise_max(mx, some);
      }
      __syncthreads();                 // K of the first tile has been read
    }
    // Holds: K of tile t + 1 and V^T of tile t in LDS, the scores of tile t in sc.
    auto step = [&](int t, f32x16 (&sc)[2], f32x16 (&sn)[2]) {
      const bool more = t + 1 < t_end;
      int s3 = 0;
      if (t + 2 < t_end) load_k(t + 2, s2);
      if (more) load_v(t + 1, s1);
      s3 = slot_of(min(t + 3, t_end - 1));
      const uint64_t next_keys = there64(t + 1, s1);
      if (active) {
        const float base = m == -INFINITY ? 0.f : m - kWideBias;
        const _Float16* kt = lds + k_buf(t + 1);
        const _Float16* vt = lds + v_buf(t);
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
          const f32x16 zero = {};
          sn[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k_frag(kt, i), q[i >> 1], i < 2 ? zero : sn[i & 1], 0, 0, 0);
#pragma unroll
          for (int e = 0; e < 8 / KS; ++e) weight(sc, i * (8 / KS) + e, base);
        }
        bool some = true;
        if (more && (~next_keys || (t + 1) * kTile + kTile > s.len)) some = mask_scores(sn, t + 1, next_keys);
        float mx = -INFINITY;
#pragma unroll
        for (int grp = 0; grp < 4; ++grp)
#pragma unroll
          for (int i = 0; i < TN; ++i) {
            const f16x8 v = v_frag(vt, grp, i);
            o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, hi[grp], o[i], 0, 0, 0);
            o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, lo[grp], o[i], 0, 0, 0);
            if (grp < 2) {
#pragma unroll
              for (int e = 0; e < 8 / TN; ++e) weight(sc, 16 + (grp * TN + i) * (8 / TN) + e, base);
            } else {
#pragma unroll
              for (int e = 0; e < 16 / TN; ++e) {
                const int k = ((grp - 2) * TN + i) * (16 / TN) + e;
                mx = fmaxf(mx, sn[k >> 4][k & 15]);
              }
            }
          }
        if (more) raise_max(mx, some);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (more && ~next_keys) mend_v(t + 1, next_keys);
      s1 = s2;
      s2 = s3;
      __syncthreads();
    };
    int t = p.t0;
    for (; t + 1 < t_end; t += 2) {
      step(t, sa, sb);
      step(t + 1, sb, sa);
    }
    if (t < t_end) step(t, sa, sb);

    l += __shfl_xor(l, 32);
    bool finite = fabsf(l) < INFINITY;
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) finite &= fabsf(o[t][r]) < INFINITY;
    const bool bad = __any(!finite);
    if (!there) continue;
    const int64_t row = (int64_t)(s.first + node) * a.nq + head;
    if (p.t0 == 0 && p.t1 == s.units) {
      const float inv = m == -INFINITY ? 0.f : 1.0f / l;
      _Float16* out = a.out + row * HD + 4 * half;
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<f16x4*>(out + t * 32 + 8 * r) = f16x4{(_Float16)(o[t][4 * r] * inv), (_Float16)(o[t][4 * r + 1] * inv),
                                                                  (_Float16)(o[t][4 * r + 2] * inv), (_Float16)(o[t][4 * r + 3] * inv)};
      if (half == 0) a.again[row] = bad;
    } else {
      const int64_t e0 = (int64_t)(2 * g + (p.t0 == 0)) * R + w * 32 + col;
      if (half == 0) a.ml[e0] = make_float2(bad ? NAN : m, l);
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<f32x4*>(a.part + e0 * HD + t * 32 + 8 * r + 4 * half) = f32x4{o[t][4 * r], o[t][4 * r + 1], o[t][4 * r + 2], o[t][4 * r + 3]};
    }
  }
}

// ---- joining
// One (row, query head) alone, over the keys that it sees, 256 at a time: a
// thread a score, then a thread a dimension of every (256 / HD)-th value.
template <int HD>
__device__ __forceinline__ void row_again(const AttnTree& a, const Seq& s, int b, int r, int hq, float* s_p, float* s_red) {
  constexpr int PARTS = 256 / HD;
  const int t = threadIdx.x, h = hq / a.group, node = r - s.first, dkv = a.nkv * HD, d = t % HD, part = t / HD;
  const uint32_t* words = a.mask + (int64_t)r * a.mask_words;
  const int32_t* table = a.table + (int64_t)b * a.n_table;
  const _Float16* q = a.q + ((int64_t)r * a.nq + hq) * HD;
  float m = -INFINITY, l = 0.f, acc = 0.f;
  for (int j0 = 0; j0 < s.keys; j0 += 256) {
    const int j = j0 + t, slot = j < s.keys ? table[j >> a.cshift] : -1;
    const bool on = (unsigned)slot < (unsigned)a.n_slots && sees(a, s, j, node, words);
    float score = -INFINITY, top = -INFINITY;
    if (on) {
      const _Float16* k = reinterpret_cast<const _Float16*>(a.slab + slot * a.slot_bytes) + (int64_t)(j & (a.C - 1)) * dkv + h * HD;
      float sum = 0.f;
      for (int e = 0; e < HD; ++e) sum = __builtin_fmaf((float)k[e], (float)q[e], sum);
      score = sum * a.scale_log2;
      top = fmaxf(score, kLowest);
    }
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
    __syncthreads();                   // the keys before have been read
    if ((t & 63) == 0) s_red[t >> 6] = top;
    __syncthreads();
    const float now = fmaxf(fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])), m);
    const float alpha = now == m ? 1.f : exp2_hw(m - now);
    m = now;
    s_p[t] = on ? exp2_hw(score - m) : -1.f;      // -1: not seen
    l *= alpha;
    acc *= alpha;
    __syncthreads();
    for (int k = part; k < 256; k += PARTS) {
      const float p = s_p[k];
      if (p == -1.f) continue;
      const int jk = j0 + k;
      const _Float16* v = reinterpret_cast<const _Float16*>(a.slab + table[jk >> a.cshift] * a.slot_bytes) + (int64_t)a.C * dkv +
                          (int64_t)(h * HD + d) * a.C + (jk & (a.C - 1));
      acc = __builtin_fmaf(p, (float)*v, acc);
      l += p;
    }
  }
  __syncthreads();
  s_p[t] = acc;
  if (d == 0) s_red[part] = l;
  __syncthreads();
  if (part == 0) {
    float sum = 0.f, den = 0.f;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      sum += s_p[k * HD + d];
      den += s_red[k];
    }
    a.out[((int64_t)r * a.nq + hq) * HD + d] = (_Float16)(m == -INFINITY ? 0.f : sum / den);
  }
}

// Joins the partials of one (row, query head): those of workgroups g0 .. g1.
// Group pg of LPP lanes takes partials pg, pg + NG, ... with their own running
// max, four dimensions a lane, and the groups meet in LDS; a partial's max, sum
// and values come in one trip to memory.  What had sums that are not finite is
// taken again.
template <int HD, int R, int UNIT>
__global__ __launch_bounds__(256) void tree_join_kernel(AttnTree a) {
  constexpr int LPP = HD / 4, NG = 256 / LPP, AHEAD = 4;     // lanes per partial, partials at once
  __shared__ float s_m[NG], s_l[NG];
  __shared__ f32x4 s_acc[NG][LPP];
  const int r = blockIdx.x / a.nq, hq = blockIdx.x % a.nq, h = hq / a.group;
  const int b = a.row_seq[r];
  if (b < 0) return;
  const Seq s = seq_of<R, UNIT>(a, b);
  const int n_units = a.base[a.n_seq] * a.nkv, x = (r - s.first) * a.group + hq - h * a.group, tile = x / R, c = x - tile * R;
  const int t = threadIdx.x, dl = t % LPP, pg = t / LPP;
  const int nw = shares(a, n_units), f0 = a.base[b] * a.nkv + (h * s.tiles + tile) * s.units;
  const int g0 = share_of(f0, nw, n_units), n = share_of(f0 + s.units - 1, nw, n_units) - g0 + 1;
  bool again = false;
  if (n == 1) {                                    // written whole
    if (!a.again[blockIdx.x]) return;
    again = true;
  }
  auto part = [&](int i) { return (int64_t)(2 * (g0 + i) + (i == 0)) * R + c; };
  float m = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (n > 1)
    for (int i0 = pg; i0 < n; i0 += AHEAD * NG) {
      float2 ml[AHEAD];
      f32x4 v[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int64_t at = part(min(i0 + k * NG, n - 1));
        ml[k] = a.ml[at];
        v[k] = *reinterpret_cast<const f32x4*>(a.part + at * HD + dl * 4);
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        if (i0 + k * NG >= n || ml[k].x == -INFINITY) continue;      // no key seen
        again |= ml[k].x != ml[k].x;
        const float top = fmaxf(m, ml[k].x), old = m == top ? 1.f : exp2_hw(m - top), wt = exp2_hw(ml[k].x - top);
        m = top;
        l = l * old + wt * ml[k].y;
        acc = acc * old + v[k] * wt;
      }
    }
  if (__syncthreads_or(again)) {
    row_again<HD>(a, s, b, r, hq, reinterpret_cast<float*>(s_acc), s_m);
    return;
  }
  if (dl == 0) {
    s_m[pg] = m;
    s_l[pg] = l;
  }
  s_acc[pg][dl] = acc;
  __syncthreads();
  if (pg == 0) {
    float top = -INFINITY, den = 0.f;
#pragma unroll
    for (int i = 0; i < NG; ++i) top = fmaxf(top, s_m[i]);
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const float wt = s_m[i] == -INFINITY ? 0.f : exp2_hw(s_m[i] - top);
      den += wt * s_l[i];
      acc += s_acc[i][dl] * wt;
    }
    const float inv = top == -INFINITY ? 0.f : 1.0f / den;
    *(reinterpret_cast<f16x4*>(a.out + (int64_t)blockIdx.x * HD) + dl) =
        f16x4{(_Float16)(acc[0] * inv), (_Float16)(acc[1] * inv), (_Float16)(acc[2] * inv), (_Float16)(acc[3] * inv)};
  }
}

int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

// Columns of a tile for `cols` columns of an average sequence.
int tile_cols(int64_t cols) { return cols <= 16 ? 16 : cols <= 32 ? 32 : cols <= 64 ? 64 : cols <= 128 ? 128 : 256; }

int most_shares(int R) { return R <= 32 ? kFewWgs : 256 * kWideWaves * 32 / R > 512 ? 512 : 256 * kWideWaves * 32 / R; }

template <int HD, int R>
void launch(const AttnTree& a, hipStream_t s) {
  constexpr int UNIT = R <= 32 ? kFewUnit : kTile;
  const dim3 grid(a.wgs);
  if constexpr (R <= 32) {
    if (a.C < kBlock)
      hipLaunchKernelGGL((tree_few_kernel<HD, R / kCols, true>), grid, dim3(64 * kFewWaves), 0, s, a);
    else
      hipLaunchKernelGGL((tree_few_kernel<HD, R / kCols, false>), grid, dim3(64 * kFewWaves), 0, s, a);
  } else {
    if (a.C < kTile)
      hipLaunchKernelGGL((tree_wide_kernel<HD, R / 32, true>), grid, dim3(2 * R), 0, s, a);
    else
      hipLaunchKernelGGL((tree_wide_kernel<HD, R / 32, false>), grid, dim3(2 * R), 0, s, a);
  }
  hipLaunchKernelGGL((tree_join_kernel<HD, R, UNIT>), dim3(a.m * a.nq), dim3(256), 0, s, a);
}

template <int HD>
void launch(const AttnTree& a, int R, hipStream_t s) {
  if (R == 16) launch<HD, 16>(a, s);
  if (R == 32) launch<HD, 32>(a, s);
  if (R == 64) launch<HD, 64>(a, s);
  if (R == 128) launch<HD, 128>(a, s);
  if (R == 256) launch<HD, 256>(a, s);
}

}  // namespace

int64_t attention_tree_units(int m, int n_seq, int n_table, int chunk_tokens, int nq, int nkv) {
  const int64_t units = ((int64_t)n_table * chunk_tokens + kTile - 1) / kTile;
  const int64_t tiles = ((int64_t)m * (nq / nkv) + 15) / 16 + n_seq;
  return tiles * nkv * units;
}

// Partials for the widest tile that fewer sequences of these rows may take, so that one workspace serves them too.
int64_t attention_tree_ws_bytes(int m, int n_seq, int nq, int nkv, int hd) {
  int64_t cols = 0;
  for (int R = 16; R <= tile_cols((int64_t)m * (nq / nkv)); R *= 2) cols = std::max<int64_t>(cols, (int64_t)2 * most_shares(R) * R);
  return up256(((int64_t)n_seq + 1) * 4) + up256((int64_t)m * 4) + up256((int64_t)m * nq) + up256(cols * 8) + cols * hd * 4;
}

void launch_attention_tree(AttnTree a, int hd, void* ws, hipStream_t s) {
  const int R = tile_cols(((int64_t)a.m + a.n_seq - 1) / a.n_seq * a.group);
  uint8_t* p = reinterpret_cast<uint8_t*>(ws);
  a.base = reinterpret_cast<int32_t*>(p);
  p += up256(((int64_t)a.n_seq + 1) * 4);
  a.row_seq = reinterpret_cast<int32_t*>(p);
  p += up256((int64_t)a.m * 4);
  a.again = p;
  p += up256((int64_t)a.m * a.nq);
  a.ml = reinterpret_cast<float2*>(p);
  p += up256((int64_t)2 * most_shares(R) * R * 8);
  a.part = reinterpret_cast<float*>(p);
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)hd);
  const int64_t most = attention_tree_units(a.m, a.n_seq, a.n_table, a.C, a.nq, a.nkv);
  a.wgs = most < most_shares(R) ? (int)most : most_shares(R);
  if (hd == 128)
    launch<128>(a, R, s);
  else
    launch<64>(a, R, s);
}

}  // namespace mzk
