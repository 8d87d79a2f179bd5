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
// infinite or NaN: then sums that are not finite show it, and the columns that
// they belong to, and no others, are taken again, a (row, head) at a time, with fp32
// products of what the row sees alone.
#include <algorithm>

#include "mz_kernels.h"

namespace mzk {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kCus = 256, kShares = 512;      // most shares: two workgroups a CU
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

// Shares of `total` units: as many as there are workgroups, but of a.least units
// at least, or where those are too few for the CUs, of a.fewest.  Each share costs
// a start and fp32 partials (32 ragged sequences: offsets and shares are known 3.9 us
// after the launch, queries, table and first tile are there after 9.7, its scores after
// 10.7): tiles of 128 columns want 8 units (8 ragged sequences of up to 4096 keys 40.8 us; at least 4:
// 44.6; 8 of 26 nodes at 4096 keys 58, at least 12: 66), and 3 where one tree is all there
// is (26 nodes at 2048 keys 15.5 us; 1: 16.4, 2: 17.0, 4: 19.3).
__device__ __forceinline__ int shares(const AttnTree& a, int total) {
  return max(1, min(a.wgs, max(total / a.least, min(kCus, total / a.fewest))));
}

// The workgroup whose share [g total / nw, (g + 1) total / nw) holds unit u.
__device__ __forceinline__ int share_of(int u, int nw, int total) {
  return (int)((((uint64_t)u + 1) * nw - 1) / (unsigned)total);
}

// Inclusive sum over the 64 NW threads; sum: of all, below 0 where any of them is bad.
template <int NW>
__device__ __forceinline__ int block_scan(int v, bool bad, int* red, int& sum) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  const bool any_bad = __any(bad);
  __syncthreads();
  if (lane == 63) red[w] = any_bad ? -1 : v;
  __syncthreads();
  int before = 0, top = 0;
  sum = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    if (i < w) before += red[i];
    sum += red[i];
    top |= red[i];
  }
  if (top < 0) sum = -1;
  return v + before;
}

// A workgroup's share [u, end) of the units, and the sequence that it begins
// in, whose units begin at `first`.  On the way, for the second kernel, of every row
// its sequence's first unit, units (0: none has the row), tiles and first row: each
// workgroup writes those of some sequences.  (Every workgroup looks through all sequences:
// 1.6 ms for 2^18 of them, nearly all without rows.)  s: NT + NW + 2 ints in LDS.
//
// The number of units fits 31 bits because the sequences' rows are m at most, which
// holds for offsets that ascend only: with others the sums below could pass 31 bits,
// and shares begin where no sequence is.  One pair that descends leaves no units at all.
struct Share {
  int u, end, b, first;
};
template <int R, int UNIT, int NW>
__device__ __forceinline__ bool share_begin(const AttnTree& a, int* s_all, Share& sh) {
  constexpr int NT = 64 * NW;
  int *s_base = s_all, *s_red = s_all + NT, *s_at = s_red + NW;
  if (blockIdx.x == gridDim.x - 1) {
    const int before = min(max(a.row_off[0], 0), a.m), behind = min(max(a.row_off[a.n_seq], before), a.m);
    for (int i = threadIdx.x; i < before + a.m - behind; i += NT) a.rows[i < before ? i : behind + i - before] = make_int4(0, 0, 0, 0);
  }
  int total = 0, u_mine = 0, u_before = 0;
  bool bad = false;
  auto units = [&](int b) {
    if (b >= a.n_seq) return 0;
    const Seq s = seq_of<R, UNIT>(a, b);
    bad |= min(max(a.row_off[b + 1], 0), a.m) < s.first;
    return s.tiles * s.units;
  };
  for (int b0 = 0; b0 < a.n_seq; b0 += NT) {
    u_mine = units(b0 + threadIdx.x);
    int sum;
    u_before = total + block_scan<NW>(u_mine, bad, s_red, sum) - u_mine;
    if (sum < 0) {
      total = 0;
      break;
    }
    total += sum;
    s_base[threadIdx.x] = u_before;
    __syncthreads();
    const int grid = gridDim.x, skip = (int)((blockIdx.x + (unsigned)grid - (unsigned)(b0 % grid)) % grid);
    for (int b = b0 + skip; b < min(b0 + NT, a.n_seq); b += grid) {
      const Seq s = seq_of<R, UNIT>(a, b);
      const int end = min(max(a.row_off[b + 1], s.first), a.m);
      for (int r = s.first + threadIdx.x; r < end; r += NT)
        a.rows[r] = make_int4(s_base[b - b0] * a.nkv, r - s.first < s.nodes ? s.units : 0, s.tiles, s.first);
    }
  }
  const int n_units = total * a.nkv, nw = shares(a, n_units), g = blockIdx.x;
  if (g == 0 && threadIdx.x == 0) *a.total = n_units;
  if (g >= nw || n_units == 0) return false;      // (no units: no sequence to begin in)
  sh.u = __builtin_amdgcn_readfirstlane((int)((uint64_t)g * n_units / nw));
  sh.end = __builtin_amdgcn_readfirstlane((int)(((uint64_t)g + 1) * n_units / nw));
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
      u_before = run + block_scan<NW>(u_mine, false, s_red, sum) - u_mine;
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

// One (row, query head) alone, over the keys that it sees, NT at a time: a
// thread a score, then a thread a dimension of every (NT / HD)-th value.  s_p: NT
// floats in LDS, s_red: max(NT / 64, NT / HD).
template <int HD, int NT>
__device__ __forceinline__ void row_again(const AttnTree& a, const Seq& s, int b, int r, int hq, float* s_p, float* s_red) {
  constexpr int PARTS = NT / HD;
  const int t = threadIdx.x, h = hq / a.group, node = r - s.first, dkv = a.nkv * HD, d = t % HD, part = t / HD;
  const uint32_t* words = a.mask + (int64_t)r * a.mask_words;
  const int32_t* table = a.table + (int64_t)b * a.n_table;
  const _Float16* q = a.q + ((int64_t)r * a.nq + hq) * HD;
  float m = -INFINITY, l = 0.f, acc = 0.f;
  for (int j0 = 0; j0 < s.keys; j0 += NT) {
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
    float now = m;
#pragma unroll
    for (int x = 0; x < NT / 64; ++x) now = fmaxf(now, s_red[x]);
    const float alpha = now == m ? 1.f : exp2_hw(m - now);
    m = now;
    s_p[t] = on ? exp2_hw(score - m) : -1.f;      // -1: not seen
    l *= alpha;
    acc *= alpha;
    __syncthreads();
    for (int k = part; k < NT; k += PARTS) {
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
  __syncthreads();
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
//
// Bound by the chain of a share: offsets, table, keys, one trip to memory each, then
// the waves' sums.  One tree of 7 nodes at 2048 keys, 8 KV heads of 64 with 4 query
// heads each, 8.3 us, 4.2 MB of keys and values.
constexpr int kFewUnit = 128, kFewWaves = 4, kBlock = 32, kCols = 16;
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
  __shared__ float s_ml[kFewWaves][2][R], s_again[kFewWaves];
  __shared__ int s_all[64 * kFewWaves + kFewWaves + 2];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, lg = lane >> 4, dkv = a.nkv * HD, g = blockIdx.x;
  Share sh;
  if (!share_begin<R, UNIT, kFewWaves>(a, s_all, sh)) return;
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
      const bool whole = p.t0 == 0 && p.t1 == s.units;
      bool bad = false;                // the column's sums
      if (__syncthreads_or(!finite && i < s.nodes))
        for (int y = p.tile * R + nb * kCols, k = 0; k < kCols && y / a.group < s.nodes; ++k, ++y) {
          const int again = __syncthreads_or(!finite && c == k);
          if (c == k) bad = again;
          if (again && whole)
            row_again<HD, 64 * kFewWaves>(a, s, sh.b, s.first + y / a.group, p.h * a.group + y % a.group, &s_o[0][0][0][0], s_again);
        }
      if (i >= s.nodes || (bad && whole)) continue;
      const int64_t row = (int64_t)(s.first + i) * a.nq + head;
      if (whole) {
        typedef _Float16 out_vec __attribute__((ext_vector_type(DPT)));
        const float inv = mx == -INFINITY ? 0.f : 1.0f / den;
        out_vec y;
#pragma unroll
        for (int e = 0; e < DPT; ++e) y[e] = (_Float16)(acc[e] * inv);
        *reinterpret_cast<out_vec*>(a.out + row * HD + dbase) = y;
      } else {
        const int64_t e0 = (int64_t)(2 * g + (p.t0 == 0)) * a.cols + x;
        if (dbase == 0) a.ml[e0] = make_float2(bad ? NAN : mx, den);
#pragma unroll
        for (int e = 0; e < DPT; e += 4)
          *reinterpret_cast<float4*>(a.part + e0 * HD + dbase + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
      }
    }
  }
}

// ---- more columns
// Four waves own 32 columns each and meet the same keys, 64 at a time, which are
// loaded into LDS once for all of them (global_load_lds, 16 bytes a lane, one
// tile ahead): S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16.  Lane l
// feeds row / column l % 32 with the 8 consecutive k of group l / 32; element r
// of the sums is row 8 (r / 4) + 4 (l / 32) + r % 4.  The score product's row i holds
// the key whose bits 2 and 3 are those of i exchanged, so that a lane's scores are
// eight consecutive keys from 16 g + 8 (l / 32) on, g = 0..3, and the P operand meets
// 16-byte runs of V^T.
//
// A step multiplies the scores of tile t + 1, then P V of tile t.  The weights of
// tile t are formed under the products up to those that need them, the max of
// tile t + 1 under P V.  The running max is raised only where a tile exceeds it by
// more than kSlack, so that sums are seldom scaled.  Slots come from a copy of the
// next kWindow tiles' stretch of the chunk table in LDS: a read of the table between
// the loads would wait for them.
//
// Measured: 4 sequences of 24576 keys and 64 nodes, 8 KV heads of 128 with 4 query
// heads each, 170 us call after call, 164-212 as the clock goes where a profiler lies
// between the calls: 155 GFLOP with the weights' lower halves, 122 us at the rate of a
// large f16 product (the matrix units are busy 51 % of the cycles, at 1.7 GHz), loads
// alone 90.  (The last step of a piece multiplies scores that nobody uses, one
// tile's K Q^T in 8 or more.)  All 256 registers are taken; 20 bytes a lane (SMALL: 56)
// go to scratch before a piece's loop and come back after it.  One workgroup of 256 columns a CU,
// which reads each key once, not twice, takes as long (184 for 187), and longer where
// trees are smaller (32 ragged 129 for 101).  32 ragged sequences of up to 8192 keys and 16
// nodes 90: 373 MB, loads alone 83.
constexpr int kTile = 64, kWideWaves = 4;
constexpr float kSlack = 4.f, kWideBias = 11.f;
constexpr int kWindow = 64;

// LDS tiles are swizzled on 16-byte columns: row r's column c lies at c ^ r % 16
// (256-byte rows), c ^ (r / 2) % 8 (128-byte rows), so that neither the reads of 32
// rows' same column nor the writes of whole rows meet in a bank.
template <int HALVES>
__device__ __forceinline__ int swizzle(int r, int c) {
  return HALVES == 128 ? c ^ (r & 15) : c ^ ((r >> 1) & 7);
}
template <int HALVES>
__device__ __forceinline__ int tile_at(int r, int c) { return r * HALVES + swizzle<HALVES>(r, c) * 8; }

__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// SMALL: chunks of fewer tokens than a tile.
template <int HD, bool SMALL>
__global__ __launch_bounds__(64 * kWideWaves, 2) void tree_wide_kernel(AttnTree a) {
  constexpr int NW = kWideWaves, R = 32 * NW, KT = kTile, UNIT = KT;
  constexpr int KC = HD / 8, VC = KT / 8;                      // 16-byte columns of a key, of a dimension
  constexpr int PER = KT * KC / 64 / NW;                       // stretches of 1 KB, 64 lanes' 16 bytes, of a tile and a wave
  constexpr int TILE = KT * HD;                                // halves
  constexpr int KS = HD / 16, TN = HD / 32;
  __shared__ __attribute__((aligned(16))) _Float16 lds[4 * TILE];      // K of two tiles, V^T of two
  __shared__ int window[SMALL ? kWindow * KT / 8 + 1 : kWindow + 1];
  __shared__ float s_again[NW];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5, dkv = a.nkv * HD, g = blockIdx.x;
  Share sh;
  if (!share_begin<R, UNIT, NW>(a, reinterpret_cast<int*>(lds), sh)) return;

  // where the lane's 16 bytes of a stretch come from: stretch i NW + w holds
  // pieces 64 (i NW + w) + lane of the swizzled tile, so that from one i to the next
  // the key (K) or the dimension (V^T) goes on by a multiple of 16, and the column
  // stays as it is
  constexpr int K_STEP = NW * 64 / KC, V_STEP = NW * 64 / VC;
  const int k_row = (w * 64 + lane) / KC, v_row = (w * 64 + lane) / VC;
  const unsigned k_of = swizzle<HD>(k_row, lane % KC) * 16u;
  const int v_key = swizzle<KT>(v_row, lane % VC) * 8;         // the first of the eight keys
  static_assert(PER >= 1 && V_STEP % 16 == 0 && K_STEP % 16 == 0, "columns of the stretches");
  typedef __attribute__((address_space(3))) void lds_void;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)lds);
  // 64 lanes' 16 bytes from `from`, or from a base in scalar registers + at, into
  // LDS.  (Wait states lie between the write of M0, and a vector instruction's of the
  // base, and the load that reads them.)
  auto fetch = [&](const uint8_t* from, int to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds0 + to * 2), "v"(from) : "memory", "m0");
  };
  auto fetch_from = [&](uint64_t base, unsigned at, int to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds0 + to * 2), "v"(at), "s"(base) : "memory", "m0");
  };

  Seq s = seq_of<R, UNIT>(a, sh.b);
  while (sh.u < sh.end) {
    const Piece p = next_piece<R, UNIT>(a, sh, s);
    const int32_t* table = a.table + (int64_t)sh.b * a.n_table;
    const int last = s.keys - 1, t_end = p.t1;
    const int x = p.tile * R + w * 32 + col, node = x / a.group, head = p.h * a.group + x - node * a.group;
    const bool there = node < s.nodes;
    const bool active = (p.tile * R + w * 32) / a.group < s.nodes;      // of the wave
    const uint32_t* words = a.mask + (int64_t)(s.first + (there ? node : 0)) * a.mask_words;

    // The table's stretch of tiles w0 .. w0 + kWindow - 1.
    int w0 = p.t0, c0 = 0;
    auto fill_window = [&](int t) {
      w0 = t;
      c0 = (t * KT) >> a.cshift;
      const int n = min(((t + kWindow) * KT - 1) >> a.cshift, last >> a.cshift) - c0 + 1;
      for (int i = threadIdx.x; i < n; i += 64 * NW) window[i] = table[c0 + i];
      __syncthreads();
    };
    // The slot of key j of the window's tiles (keys past the last one: its slot).
    auto slot_at = [&](int j) { return window[(min(j, last) >> a.cshift) - c0]; };
    auto clean = [&](int slot) { return (unsigned)slot < (unsigned)a.n_slots ? slot : 0; };
    // Slots are read a step before they are used: with SMALL those of what the lane
    // loads, else the tile's, into scalar registers, those of tiles t + 1 and t + 2 at step t.
    constexpr int KSLOTS = SMALL ? PER : 1;
    int k_slot[KSLOTS], v_slot = 0, slot1, slot2;
    const unsigned k_lane = (unsigned)k_row * (unsigned)dkv * 2u + p.h * HD * 2u + k_of;
    const unsigned v_lane = ((unsigned)(dkv + p.h * HD + v_row) * (unsigned)a.C + v_key) * 2u;
    const uint64_t slab = (uint64_t)(uintptr_t)a.slab;
    auto scalar_slot = [&](int t) { return __builtin_amdgcn_readfirstlane(slot_at(min(t, t_end - 1) * KT)); };
    auto load_k = [&](int t, int slot) {
      const int j0 = (t * KT) & (a.C - 1), to = (t & 1) * TILE + w * 512;
      const uint64_t base = slab + (uint64_t)clean(slot) * (uint64_t)a.slot_bytes + (unsigned)j0 * (unsigned)dkv * 2u;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if constexpr (SMALL) {
          const int row = k_row + i * K_STEP;
          fetch(a.slab + (int64_t)clean(k_slot[i]) * a.slot_bytes + ((unsigned)((j0 + row) & (a.C - 1)) * (unsigned)dkv * 2u + p.h * HD * 2u + k_of),
                to + i * NW * 512);
        } else {
          fetch_from(base + (unsigned)(i * K_STEP) * (unsigned)dkv * 2u, k_lane, to + i * NW * 512);
        }
      }
    };
    auto load_v = [&](int t, int slot) {
      const int j0 = (t * KT) & (a.C - 1), to = (2 + (t & 1)) * TILE + w * 512;
      const uint64_t base = slab + (uint64_t)clean(slot) * (uint64_t)a.slot_bytes + (unsigned)j0 * 2u;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if constexpr (SMALL)
          fetch(a.slab + (int64_t)clean(v_slot) * a.slot_bytes +
                    ((unsigned)(dkv + p.h * HD + v_row + i * V_STEP) * (unsigned)a.C + (unsigned)((j0 + v_key) & (a.C - 1))) * 2u,
                to + i * NW * 512);
        else
          fetch_from(base + (unsigned)(i * V_STEP) * (unsigned)a.C * 2u, v_lane, to + i * NW * 512);
      }
    };
    auto slots_of_k = [&](int t) {
      if constexpr (SMALL)
#pragma unroll
        for (int i = 0; i < KSLOTS; ++i) k_slot[i] = slot_at(t * KT + k_row + i * K_STEP);
    };
    auto slots_of_v = [&](int t) {
      if constexpr (SMALL) v_slot = slot_at(t * KT + v_key);
    };
    // Keys of tile t that are there, and zeros for the values of the others.
    auto there64 = [&](int t, int slot) -> uint64_t {
      if constexpr (SMALL) {
        const int j = t * KT + lane;
        return __ballot((unsigned)slot_at(j) < (unsigned)a.n_slots && j < s.keys);
      } else {
        return (unsigned)slot < (unsigned)a.n_slots ? ones64(s.keys - t * KT) : 0;
      }
    };
    auto mend_v = [&](int t, uint64_t keys) {
      const unsigned on = (unsigned)(keys >> v_key) & 0xFF;
      if (on == 0xFF) return;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        f16x8* v = reinterpret_cast<f16x8*>(lds + (2 + (t & 1)) * TILE + (i * NW + w) * 512 + lane * 8);
        f16x8 e = *v;
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = (on >> k) & 1 ? e[k] : (_Float16)0.f;
        *v = e;
      }
    };

    f16x8 q[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      q[ks] = f16x8{};
      if (there) q[ks] = *reinterpret_cast<const f16x8*>(a.q + ((int64_t)(s.first + node) * a.nq + head) * HD + ks * 16 + half * 8);
    }
    __syncthreads();                   // the piece before has been read
    fill_window(p.t0);
    const int slot0 = SMALL ? 0 : scalar_slot(p.t0);
    slot1 = SMALL ? 0 : scalar_slot(p.t0 + 1);
    slot2 = SMALL ? 0 : scalar_slot(p.t0 + 2);
    slots_of_k(p.t0);
    slots_of_v(p.t0);
    load_k(p.t0, slot0);
    load_v(p.t0, slot0);
    if (p.t0 + 1 < t_end) {
      slots_of_k(p.t0 + 1);
      load_k(p.t0 + 1, slot1);
    }
    f32x16 o[TN];
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
    float m = -INFINITY, l = 0.f;

    const int krow = (col & ~12) | ((col & 8) >> 1) | ((col & 4) << 1);
    auto k_frag = [&](const _Float16* k, int i) {        // of score product i
      return *reinterpret_cast<const f16x8*>(&k[tile_at<HD>((i & 1) * 32 + krow, (i >> 1) * 2 + half)]);
    };
    auto v_frag = [&](const _Float16* v, int grp, int t) {
      return *reinterpret_cast<const f16x8*>(&v[tile_at<KT>(t * 32 + col, grp * 2 + half)]);
    };
    // Scores of tile t that do not count become -inf; keys: those that are there.
    auto mask_scores = [&](f32x16 (&sc)[2], int t, uint64_t keys) {
      const uint64_t on = keys & seen64(a, s, t * KT, node, words);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const unsigned mine = (unsigned)(on >> (32 * kk + 8 * half));
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float v = sc[kk][r];
          sc[kk][r] = (mine >> (16 * (r >> 3) + (r & 7))) & 1 ? v : -INFINITY;
        }
      }
      return on != 0;
    };
    // The max of a column's scores is the lane's and lane ^ 32's.  A tile with a key
    // that counts raises it to at least the lowest fp32 value, so -inf means that
    // none was seen.
    auto raise_max = [&](float mx, float other, bool some) {
      mx = fmaxf(mx, other) * a.scale_log2;
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
    f16x2 hi[16], lo[16];      // of two scores each, four to a P operand
    float e0 = 0.f, e1 = 0.f, base = 0.f;
    // The weights of scores 2 i and 2 i + 1 in four parts of about the same time
    // (j = 4 i + part), so that they fit under products: the exponentials; their sum;
    // their halves, lo = f16(e - hi) in one instruction each.  (Its inputs are a
    // conversion's, not an exponential's or a product's, and a product may read it
    // two wait states later.)
    auto weigh = [&](const f32x16 (&sc)[2], int j) {
      const int i = j >> 2;
      if ((j & 3) == 0) e0 = exp2_hw(__builtin_fmaf(sc[i >> 3][2 * (i & 7)], a.scale_log2, -base));
      if ((j & 3) == 1) e1 = exp2_hw(__builtin_fmaf(sc[i >> 3][2 * (i & 7) + 1], a.scale_log2, -base));
      if ((j & 3) == 2) {
        l += e0;
        l += e1;
        asm volatile("" : "+v"(l));
      }
      if ((j & 3) == 3) {
        hi[i] = f16x2{(_Float16)e0, (_Float16)e1};
        asm volatile("v_fma_mixlo_f16 %0, %1, -1.0, %2 op_sel:[0,0,0] op_sel_hi:[1,0,0]\n\t"
                     "v_fma_mixhi_f16 %0, %1, -1.0, %3 op_sel:[1,0,0] op_sel_hi:[1,0,0]\n\ts_nop 1"
                     : "=&v"(lo[i]) : "v"(hi[i]), "v"(e0), "v"(e1));
      }
    };
    // Product i of those before the last 16 keys' carries its share of the parts,
    // so that a P operand is there when its products begin.
    constexpr int PARTS = 64, CARRY = 2 * KS + 3 * 2 * TN;
    auto carry = [&](const f32x16 (&sc)[2], int i) {
#pragma unroll
      for (int j = i * PARTS / CARRY; j < (i + 1) * PARTS / CARRY; ++j) weigh(sc, j);
    };
    auto operand = [&](const f16x2* x, int grp) {
      f16x8 y;
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = x[4 * grp + k / 2][k & 1];
      return y;
    };

    f32x16 sa[2], sb[2];
    {
      wait_loads();
      const uint64_t keys = there64(p.t0, slot0);
      if (~keys) mend_v(p.t0, keys);
      __syncthreads();
      if (active) {
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
          const f32x16 zero = {};
          sa[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k_frag(lds + (p.t0 & 1) * TILE, i), q[i >> 1], i < 2 ? zero : sa[i & 1], 0, 0, 0);
        }
        bool some = true;
        if (~keys || p.t0 * KT + KT > s.len) some = mask_scores(sa, p.t0, keys);
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 32; ++i) mx = fmaxf(mx, sa[i >> 4][i & 15]);
        raise_max(mx, __shfl_xor(mx, 32), some);
      }
      __syncthreads();                 // K of the first tile has been read
    }
    uint64_t next_keys = 0;
    int new_slot = 0;
    auto look_ahead = [&](int t) {     // what step t needs of the table
      if constexpr (SMALL) {
        if (t + 1 < t_end) slots_of_v(t + 1);
        if (t + 2 < t_end) slots_of_k(t + 2);
        if (t + 1 < t_end) next_keys = there64(t + 1, 0);
      } else {
        new_slot = slot_at(min(t + 2, t_end - 1) * KT);
      }
    };
    if constexpr (SMALL) look_ahead(p.t0);
    // Holds: K of tile t + 1 and V^T of tile t in LDS, the scores of tile t in
    // sc.  Products and what is done under each are kept in this order by
    // fences; fragments are read three products (K) and a pair of them (V^T) ahead.
    auto step = [&](int t, f32x16 (&sc)[2], f32x16 (&sn)[2]) {
      const bool more = t + 1 < t_end;
      const _Float16* kt = lds + ((t + 1) & 1) * TILE;
      const _Float16* vt = lds + (2 + (t & 1)) * TILE;
      f16x8 k0 = k_frag(kt, 0), k1 = k_frag(kt, 1), k2 = k_frag(kt, 2);
      if (more) load_v(t + 1, slot1);
      if (t + 2 < t_end) load_k(t + 2, slot2);
      const uint64_t keys = SMALL ? next_keys : there64(t + 1, slot1);
      const bool refill = t + 3 >= w0 + kWindow && t + 2 < t_end;
      if (!refill) look_ahead(t + 1);
      if (active) {
        base = m == -INFINITY ? 0.f : m - kWideBias;
        f16x8 v0, v1;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
          const f32x16 zero = {};
          const f16x8 k3 = i + 3 < 2 * KS ? k_frag(kt, i + 3) : k2;
          if (i == 2 * KS - 3) v0 = v_frag(vt, 0, 0);
          if (i == 2 * KS - 2) v1 = v_frag(vt, 0, 1);
          __builtin_amdgcn_sched_barrier(0);
          sn[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k0, q[i >> 1], i < 2 ? zero : sn[i & 1], 0, 0, 0);
          k0 = k1;
          k1 = k2;
          k2 = k3;
          carry(sc, i);
          __builtin_amdgcn_sched_barrier(0);
        }
        bool some = true;
        if (more && (~keys || (t + 1) * KT + KT > s.len)) some = mask_scores(sn, t + 1, keys);
        float mx = -INFINITY, other = -INFINITY;
        constexpr int PAIRS = 2 * TN;             // of V^T fragments: 16 keys, 32 dimensions each
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
          const int grp = i / (TN / 2), d = i % (TN / 2) * 2, ng = (i + 1) / (TN / 2), nd = (i + 1) % (TN / 2) * 2;
          const f16x8 v2 = i + 1 < PAIRS ? v_frag(vt, ng, nd) : v0, v3 = i + 1 < PAIRS ? v_frag(vt, ng, nd + 1) : v1;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            __builtin_amdgcn_sched_barrier(0);
            o[d + (k & 1)] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k & 1 ? v1 : v0, operand(k < 2 ? hi : lo, grp), o[d + (k & 1)], 0, 0, 0);
            const int slot = 4 * i + k;
            if (2 * KS + slot < CARRY) carry(sc, 2 * KS + slot);
            if (slot < 4 * TN)                // the max of the next scores under the first half
#pragma unroll
              for (int e = 0; e < 8 / TN; ++e) {
                const int y = slot * (8 / TN) + e;
                mx = fmaxf(mx, sn[y >> 4][y & 15]);
              }
            if (slot == 4 * TN) other = __shfl_xor(mx, 32);
            __builtin_amdgcn_sched_barrier(0);
          }
          v0 = v2;
          v1 = v3;
        }
        if (more) raise_max(mx, other, some);
      }
      wait_loads();
      if (more && ~keys) mend_v(t + 1, keys);
      __syncthreads();
      if (refill) {
        fill_window(t + 2);
        look_ahead(t + 1);
      }
      if constexpr (!SMALL) {
        slot1 = slot2;
        slot2 = __builtin_amdgcn_readfirstlane(new_slot);
      }
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
    const bool whole = p.t0 == 0 && p.t1 == s.units;
    const bool other_bad = __shfl_xor((int)!finite, 32);      // of the column's other dimensions
    const bool bad = !finite || other_bad;
    const int64_t row = (int64_t)(s.first + node) * a.nq + head;
    if (there && whole && !bad) {
      const float inv = m == -INFINITY ? 0.f : 1.0f / l;
      _Float16* out = a.out + row * HD + 4 * half;
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<f16x4*>(out + t * 32 + 8 * r) = f16x4{(_Float16)(o[t][4 * r] * inv), (_Float16)(o[t][4 * r + 1] * inv),
                                                                  (_Float16)(o[t][4 * r + 2] * inv), (_Float16)(o[t][4 * r + 3] * inv)};
    } else if (there && !whole) {
      const int64_t e0 = (int64_t)(2 * g + (p.t0 == 0)) * a.cols + w * 32 + col;
      if (half == 0) a.ml[e0] = make_float2(bad ? NAN : m, l);
#pragma unroll
      for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<f32x4*>(a.part + e0 * HD + t * 32 + 8 * r + 4 * half) = f32x4{o[t][4 * r], o[t][4 * r + 1], o[t][4 * r + 2], o[t][4 * r + 3]};
    }
    if (whole && __syncthreads_or(there && bad))
      for (int y = p.tile * R, k = 0; k < R && y / a.group < s.nodes; ++k, ++y)
        if (__syncthreads_or(bad && w * 32 + col == k))
          row_again<HD, 64 * NW>(a, s, sh.b, s.first + y / a.group, p.h * a.group + y % a.group, reinterpret_cast<float*>(lds), s_again);
  }
}

// ---- joining
// Joins the partials of every (row, query head) that several shares met, g0 ..
// g1.  TPR of a workgroup's threads take one: HD / 4 lanes a partial, four
// dimensions each, AHEAD of them in one trip to memory, and the groups of lanes meet in
// LDS.  Rows with sums that are not finite are taken again.  (4 sequences of 64 nodes,
// 34 MB of partials, 11.6 us; a workgroup a row there, or one for each share's columns, is
// slower.  Few rows of many shares want a workgroup each: 3.6-4.8 us for 7 nodes.  A row
// finds its sequence by halves: 8 of 2^18 sequences with infinite values 40 -> 3 ms.)
template <int HD, int R>
__global__ __launch_bounds__(256) void tree_join_kernel(AttnTree a) {
  constexpr int TPR = R <= 32 ? 256 : 64, ROWS = 256 / TPR, LPP = HD / 4, NG = TPR / LPP, AHEAD = R <= 32 ? 4 : 8;
  __shared__ float s_m[256 / LPP], s_l[256 / LPP];
  __shared__ f32x4 s_acc[256 / LPP][LPP];
  const int t = threadIdx.x, dl = t % LPP, group = t / LPP, pg = group % NG;
  const int64_t first = (int64_t)blockIdx.x * ROWS, at = first + t / TPR, rows = (int64_t)a.m * a.nq;
  const int total = *a.total, nw = shares(a, total);
  bool again = false;
  const int r = (int)(min(at, rows - 1) / a.nq), hq = (int)(at - (int64_t)r * a.nq), h = hq / a.group;
  const int4 row = a.rows[r];          // first unit, units, tiles, first row of its sequence
  int n = 0;
  float m = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  if (at < rows && row.y && total > 0) {      // (no units: rows is not filled where offsets descend)
    const int x = (r - row.w) * a.group + hq - h * a.group, tile = x / R, c = x - tile * R;
    const int f0 = row.x + (h * row.z + tile) * row.y, g0 = share_of(f0, nw, total);
    n = share_of(f0 + row.y - 1, nw, total) - g0 + 1;
    auto part = [&](int i) { return (int64_t)(2 * (g0 + i) + (i == 0)) * a.cols + c; };
    if (n > 1)                         // else it is written whole
      for (int i0 = pg; i0 < n; i0 += AHEAD * NG) {
        float2 ml[AHEAD];
        f32x4 v[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const int64_t y = part(min(i0 + k * NG, n - 1));
          ml[k] = a.ml[y];
          v[k] = *reinterpret_cast<const f32x4*>(a.part + y * HD + dl * 4);
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
  }
  if (ROWS == 1 && n <= 1) return;
  if (dl == 0) {
    s_m[group] = m;
    s_l[group] = l;
  }
  s_acc[group][dl] = acc;
  unsigned bad = 0;                    // a bit for each of the rows that are taken again
  if (__syncthreads_or(again))
#pragma unroll
    for (int k = 0; k < ROWS; ++k) bad |= (unsigned)(__syncthreads_or(again && t / TPR == k) != 0) << k;
  if (pg == 0 && n > 1 && !((bad >> (t / TPR)) & 1)) {
    float top = -INFINITY, den = 0.f;
#pragma unroll
    for (int i = 0; i < NG; ++i) top = fmaxf(top, s_m[group + i]);
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const float wt = s_m[group + i] == -INFINITY ? 0.f : exp2_hw(s_m[group + i] - top);
      den += wt * s_l[group + i];
      acc += s_acc[group + i][dl] * wt;
    }
    const float inv = top == -INFINITY ? 0.f : 1.0f / den;
    *(reinterpret_cast<f16x4*>(a.out + at * HD) + dl) =
        f16x4{(_Float16)(acc[0] * inv), (_Float16)(acc[1] * inv), (_Float16)(acc[2] * inv), (_Float16)(acc[3] * inv)};
  }
  if (!bad) return;
  __syncthreads();                     // the others' sums have been read
  for (int k = 0; k < ROWS; ++k) {
    if (!((bad >> k) & 1)) continue;
    const int r = (int)((first + k) / a.nq), hq = (int)(first + k - (int64_t)r * a.nq);
    int b = 0;                         // the row's sequence: the last that begins at or before it
    for (int behind = a.n_seq; behind - b > 1;) {
      const int mid = (b + behind) >> 1;
      if (a.row_off[mid] <= r)
        b = mid;
      else
        behind = mid;
    }
    row_again<HD, 256>(a, seq_of<R, 1>(a, b), b, r, hq, reinterpret_cast<float*>(s_acc), s_m);
  }
}

int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

// Columns of a tile for `cols` columns of an average sequence.  Tiles of 16 and 32
// start sooner, tiles of 128 share what they load and feed the matrix units better.
// us, with tiles of 16 / 32 / 128, sequences x nodes at keys (columns):
//   32 + 8 heads of 64:  1 x 7 at 2048 (28) 12.4 / 12.4 / 13.6, 8 x 7 at 4096 (28) 32.4 / 25.0 / 25.6,
//     64 x 4 at 2048 (16) 112 / 114 / 110, 1 x 26 at 2048 (104) 17.2 / 16.7 / 15.7,
//     1 x 60 at 8192 (240) 49.0 / 31.5 / 28.7
//   12 + 2 heads of 128:  8 x 5 at 16384 (30) 25.6 / 27.5 / 31.5, 2 x 5 at 4096 (30) 13.1 / 14.7 / 21.5,
//     8 ragged of 26 60.6 / 45.8 / 40.9
//   32 + 8 heads of 128:  4 x 5 at 1000 (20) 16.2 / 16.6 / 21.1, 32 x 5 at 4096 (20) 168 / 119 / 112,
//     16 x 8 at 4096 (32) 93.7 / 69.4 / 65.8, 8 x 26 at 4096 (104) 156 / 102 / 59,
//     4 x 64 at 24576 (256) 708 / 388 / 188
// (So not every average gets its fastest tile: 2-12 % are lost at 20-32 columns, one way
// or the other.)  What the rule does not see is how unlike the trees are; a prompt's
// piece beside sequences of one row takes narrow tiles and reads its own keys once for
// each of them (columns of the average; us again with 16 / 32 / 128):
//   32 + 8 heads of 128:  256 rows beside 63 of 1 at 4096 (20) 349 / 288 / 246,
//     512 beside 127 ragged to 8192 (20) 571 / 514 / 471
//   32 + 8 heads of 64:  256 beside 63 at 4096 (20) 179 / 158 / 169
//   32 + 8 heads of 128, beside sequences of no row:  256 and 63 at 4096 (16) 141 / 95 / 57,
//     512 and 127 at 8192 (16) 504 / 270 / 133
int tile_cols(int64_t cols) { return cols <= 16 ? 16 : cols <= 32 ? 32 : 128; }

// Columns of a partial, of a call of `cols` columns a KV head in all.
int part_cols(int R, int64_t cols) { return cols < R ? (int)cols : R; }

template <int HD, int R>
void launch(const AttnTree& a, hipStream_t s) {
  const dim3 grid(a.wgs);
  if constexpr (R <= 32) {
    if (a.C < kBlock)
      hipLaunchKernelGGL((tree_few_kernel<HD, R / kCols, true>), grid, dim3(64 * kFewWaves), 0, s, a);
    else
      hipLaunchKernelGGL((tree_few_kernel<HD, R / kCols, false>), grid, dim3(64 * kFewWaves), 0, s, a);
  } else {
    if (a.C < kTile)
      hipLaunchKernelGGL((tree_wide_kernel<HD, true>), grid, dim3(2 * R), 0, s, a);
    else
      hipLaunchKernelGGL((tree_wide_kernel<HD, false>), grid, dim3(2 * R), 0, s, a);
  }
  hipLaunchKernelGGL((tree_join_kernel<HD, R>), dim3((unsigned)(((int64_t)a.m * a.nq * (R <= 32 ? 4 : 1) + 3) / 4)), dim3(256), 0, s, a);
}

template <int HD>
void launch(const AttnTree& a, int R, hipStream_t s) {
  if (R == 16) launch<HD, 16>(a, s);
  if (R == 32) launch<HD, 32>(a, s);
  if (R == 128) launch<HD, 128>(a, s);
}

}  // namespace

int64_t attention_tree_units(int m, int n_seq, int n_table, int chunk_tokens, int nq, int nkv) {
  const int64_t units = ((int64_t)n_table * chunk_tokens + 31) / 32;
  const int64_t tiles = ((int64_t)m * (nq / nkv) + 15) / 16 + n_seq;
  return tiles * nkv * units;
}

// Partials for the widest tile that fewer sequences of these rows may take, so that one workspace serves them too.
int64_t attention_tree_ws_bytes(int m, int n_seq, int nq, int nkv, int hd) {
  const int64_t all = (int64_t)m * (nq / nkv), cols = (int64_t)2 * kShares * part_cols(tile_cols(all), all);
  return 256 + up256((int64_t)m * 16) + up256(cols * 8) + cols * hd * 4;
}

void launch_attention_tree(AttnTree a, int hd, void* ws, hipStream_t s) {
  const int R = tile_cols(((int64_t)a.m + a.n_seq - 1) / a.n_seq * a.group);
  a.cols = part_cols(R, (int64_t)a.m * a.group);
  uint8_t* p = reinterpret_cast<uint8_t*>(ws);
  a.total = reinterpret_cast<int32_t*>(p);
  p += 256;
  a.rows = reinterpret_cast<int4*>(p);
  p += up256((int64_t)a.m * 16);
  a.ml = reinterpret_cast<float2*>(p);
  p += up256((int64_t)2 * kShares * a.cols * 8);
  a.part = reinterpret_cast<float*>(p);
  a.least = R <= 32 ? 1 : 8;
  a.fewest = R <= 32 ? 1 : 3;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)hd);
  const int64_t most = attention_tree_units(a.m, a.n_seq, a.n_table, a.C, a.nq, a.nkv);
  a.wgs = most < kShares ? (int)most : kShares;
  if (hd == 128)
    launch<128>(a, R, s);
  else
    launch<64>(a, R, s);
}

}  // namespace mzk
