// Attention of several new tokens of every sequence of a batch, trees or
// chains, over its chunked KV cache (gfx950): for node i of sequence b, head h
// of KV head h / G,
//   out = sum_j w_j v_j / sum_j w_j,  w_j = 2^(s_j - max s),
//   s_j = log2(e) / sqrt(hd) q . k_j,  j < len or j = len + t, t in the node's mask.
//
// The G T query heads and nodes of a KV head are the columns of the products,
// R at a time, so that a key is read once for R of them.  As in
// attention_batch.hip the work is cut by keys, not by sequences: the units of 128
// keys of all (sequence, KV head, R columns) lie in one line, each workgroup
// takes an even share of it, and a second kernel joins what several shares
// summed, in a fixed order.
//
// A workgroup's four waves take the 32-key blocks of its share in turn, each
// for all R columns: S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_16x16x32,
// K and V^T fragments straight from the slots, 16 bytes a lane.  Row i of the
// score product holds key 8 (i / 4) + 4 t + i % 4 of the block (t: first or
// second product), so that the eight scores of a lane are eight consecutive
// keys: its mask is eight bits, and the P operand meets one 16-byte run of V^T.
//
// P goes into the product as two f16 values, hi + lo, of 2^(14 + s - max): 22
// bits of a weight (and what it holds down to 2^-38 of the largest), so that an
// output's only rounding to fewer bits is its own.  Both enter the same fp32 sums.  A
// weight of 0 removes what a node does not see, unless the value is infinite or NaN:
// then a sum that is not finite shows it, and the wave takes its blocks again
// with products in fp32 that leave those values out one by one.
#include "mz_kernels.h"

namespace mzk {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kUnit = 128;          // keys of a unit: a 32-key block for each wave
constexpr int kWaves = 4, kBlock = 32, kCols = 16;
constexpr int kWgs = 512;           // most workgroups that share the units
constexpr float kBias = 14.f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

struct Seq {
  int first, nodes, len, keys;      // rows first .. first + nodes - 1, keys before the tree and in all
  int tiles, units;                 // of R columns, of 128 keys
};
template <int R>
__device__ __forceinline__ Seq seq_of(const AttnTree& a, int b) {
  Seq s;
  s.first = min(max(a.row_off[b], 0), a.m);
  s.nodes = min(max(a.row_off[b + 1], s.first), a.m) - s.first;
  if (a.mask) s.nodes = min(s.nodes, 32 * a.mask_words);
  const int top = a.n_table << a.cshift;
  s.len = min(max(a.lens[b], 0), top);
  s.keys = s.nodes < top - s.len ? s.len + s.nodes : top;
  s.tiles = (s.nodes * a.group + R - 1) / R;
  s.units = (s.keys + kUnit - 1) / kUnit;
  return s;
}

__device__ __forceinline__ int shares(const AttnTree& a, int total) { return min(a.wgs, total); }

// The workgroup whose share [g total / nw, (g + 1) total / nw) holds unit u.
__device__ __forceinline__ int share_of(int u, int nw, int total) {
  return (int)((((uint64_t)u + 1) * nw - 1) / (unsigned)total);
}

// Inclusive sum over the 256 threads; sum: of all.
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
#pragma unroll
  for (int i = 0; i < kWaves; ++i)
    if (i < w) before += red[i];
  sum = red[0] + red[1] + red[2] + red[3];
  return v + before;
}

__device__ __forceinline__ unsigned ones(int n) { return n <= 0 ? 0u : n >= 8 ? 0xFFu : (1u << n) - 1; }

// Which of the eight keys from j on a node sees, of those before the end; t:
// the node, words: its mask.
__device__ __forceinline__ unsigned seen(const AttnTree& a, const Seq& s, int j, int t, const uint32_t* words) {
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
    m = ones(t - at + 1);
  }
  return m & ones(s.keys - j);
}

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
struct Tile {
  static constexpr int KS = HD / 32;          // 32-wide dimension steps of a score product
  static constexpr int DB = HD / 16;          // 16-dimension blocks of the output
  f16x8 q[NB][KS];
  f32x4 o[NB][DB];
  float m[NB], l[NB];
  int node[NB];                               // of the lane's columns, -1: none

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int d = 0; d < DB; ++d) o[nb][d] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[nb] = -INFINITY;
      l[nb] = 0.f;
    }
  }

  // The block's weights 2^(14 + s - max) of column block nb: e, their sum
  // added to l, o and l scaled to the running max.  A key that counts raises the
  // max to at least the lowest fp32 value, so -inf means that none was seen;
  // scores of -inf and NaN then go where the formula sends them.
  __device__ __forceinline__ void weights(const f16x8 (&ka)[2][KS], int nb, unsigned on, float scale, float (&e)[8]) {
    f32x4 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ka[t][ks], q[nb][ks], sc[t], 0, 0, 0);
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = sc[i >> 2][i & 3] * scale;
      e[i] = (on >> i) & 1 ? v : -INFINITY;
      top = (on >> i) & 1 ? fmaxf(top, fmaxf(v, -3.402823466e38f)) : top;
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
    const float base = m[nb] == -INFINITY ? 0.f : m[nb] - kBias;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e[i] = exp2_hw(e[i] - base);
      l[nb] += e[i];
    }
  }

  // This wave's blocks of the share: j0, j0 + 128, ... below j_end.  Table
  // entries are read a block ahead, so that a block waits for one trip to
  // memory, not two.  CAREFUL: values of weight 0 are left out of the sums.
  template <bool CAREFUL>
  __device__ __forceinline__ void blocks(const AttnTree& a, const Seq& s, const int32_t* table, int h, int j_begin, int j_end,
                                         const uint32_t* const (&words)[NB], int lane) {
    const int col = lane & 15, lg = lane >> 4, dkv = a.nkv * HD, last = s.keys - 1;
    clear();
    Slots next = slots_of<SMALL>(table, a.cshift, min(j_begin, last), col, lg, last);
    for (int j0 = j_begin; j0 < j_end; j0 += kUnit) {
      Slots at = next;
      next = slots_of<SMALL>(table, a.cshift, min(j0 + kUnit, last), col, lg, last);
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
      const unsigned k_at = (unsigned)((kj & (a.C - 1)) + (col & 3)) * (unsigned)dkv * 2u + (h * HD + lg * 8) * 2u;
      const unsigned v_at = (unsigned)a.C * dkv * 2u + ((unsigned)(h * HD + col) * a.C + (vj & (a.C - 1))) * 2u;
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
      if constexpr (!CAREFUL)
        if (__any(n_ok < 8)) {                    // values that are not there are not data: zero them
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 8; ++i) va[d][i] = i < n_ok ? va[d][i] : (_Float16)0.f;
        }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        unsigned on = ok && node[nb] >= 0 ? 0xFF : 0;
        if (tree && on) on = seen(a, s, vj, node[nb], words[nb]);
        float e[8];
        weights(ka, nb, on, a.scale_log2, e);
        if constexpr (!CAREFUL) {
          f16x8 hi, lo;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            hi[i] = (_Float16)e[i];
            lo[i] = (_Float16)(e[i] - (float)hi[i]);
          }
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            o[nb][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va[d], hi, o[nb][d], 0, 0, 0);
            o[nb][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va[d], lo, o[nb][d], 0, 0, 0);
          }
        } else {
          // o[d][r] of the lane is dimension 16 d + 4 lg + r of column col: its weight of key k lies in lane 16 (k / 8) + col
          for (int k = 0; k < kBlock; ++k) {
            const int j = j0 + k, from = (k >> 3) * 16 + col;
            float p = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) p = (k & 7) == i ? __shfl(e[i], from) : p;
            const bool in = (__shfl(on, from) >> (k & 7)) & 1;
            const int slot = __shfl(at.v, (k >> 3) * 16);
            if (!in) continue;
            const _Float16* v = reinterpret_cast<const _Float16*>(a.slab + slot * a.slot_bytes + (int64_t)a.C * dkv * 2) +
                                (int64_t)(h * HD + lg * 4) * a.C + (j & (a.C - 1));
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
              for (int r = 0; r < 4; ++r) o[nb][d][r] += p * (float)v[(int64_t)(d * 16 + r) * a.C];
          }
        }
      }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      l[nb] += __shfl_xor(l[nb], 16);
      l[nb] += __shfl_xor(l[nb], 32);
    }
  }

  __device__ __forceinline__ bool finite() const {
    bool f = true;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) f &= fabsf(o[nb][d][r]) < INFINITY;
    return f;
  }
};

template <int HD, int NB, bool SMALL>
__global__ __launch_bounds__(64 * kWaves, NB == 4 ? 1 : 2) void attn_tree_kernel(AttnTree a) {
  constexpr int R = NB * kCols, KS = HD / 32, DB = HD / 16;
  __shared__ float s_o[kWaves][DB][4][64];
  __shared__ float s_ml[kWaves][2][R];
  __shared__ int s_red[kWaves], s_at[2];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, lg = lane >> 4;

  // the second kernel finds a row's sequence here
  for (int b = blockIdx.x; b <= a.n_seq; b += gridDim.x) {
    if (b < a.n_seq) {
      const Seq s = seq_of<R>(a, b);
      const int end = min(max(a.row_off[b + 1], s.first), a.m);
      for (int r = s.first + threadIdx.x; r < end; r += 256) a.row_seq[r] = r - s.first < s.nodes ? b : -1;
    } else {
      const int before = min(max(a.row_off[0], 0), a.m), last = min(max(a.row_off[a.n_seq], before), a.m);
      for (int i = threadIdx.x; i < before + a.m - last; i += 256) a.row_seq[i < before ? i : last + i - before] = -1;
    }
  }

  // where this workgroup's share begins: (sequence, units of the sequences before it)
  int total = 0, u_mine = 0, u_before = 0;
  for (int b0 = 0; b0 < a.n_seq; b0 += 256) {
    const int b = b0 + threadIdx.x;
    u_mine = 0;
    if (b < a.n_seq) {
      const Seq s = seq_of<R>(a, b);
      u_mine = s.tiles * s.units;
    }
    int sum;
    u_before = total + block_scan(u_mine, s_red, sum) - u_mine;
    if (blockIdx.x == 0 && b < a.n_seq) a.base[b] = u_before;
    total += sum;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.base[a.n_seq] = total;
  const int n_units = total * a.nkv, nw = shares(a, n_units), g = blockIdx.x;
  if (g >= nw) return;
  int u = (int)((uint64_t)g * n_units / nw);
  const int u_end = (int)(((uint64_t)g + 1) * n_units / nw);
  if (a.n_seq > 256) {
    int run = 0;
    for (int b0 = 0; b0 < a.n_seq; b0 += 256) {
      const int b = b0 + threadIdx.x;
      u_mine = 0;
      if (b < a.n_seq) {
        const Seq s = seq_of<R>(a, b);
        u_mine = s.tiles * s.units;
      }
      int sum;
      u_before = run + block_scan(u_mine, s_red, sum) - u_mine;
      if (u >= u_before * a.nkv && u < (u_before + u_mine) * a.nkv) {
        s_at[0] = b;
        s_at[1] = u_before;
      }
      run += sum;
    }
  } else if (u >= u_before * a.nkv && u < (u_before + u_mine) * a.nkv) {
    s_at[0] = threadIdx.x;
    s_at[1] = u_before;
  }
  __syncthreads();
  int b = __builtin_amdgcn_readfirstlane(s_at[0]), first = __builtin_amdgcn_readfirstlane(s_at[1]) * a.nkv;

  Seq s = seq_of<R>(a, b);
  Tile<HD, NB, SMALL> t;
  while (u < u_end) {
    if (u >= first + s.tiles * s.units * a.nkv) {      // past this sequence: on to the next that has rows, 64 in a look
      first += s.tiles * s.units * a.nkv;
      uint64_t some = 0;
      for (++b; !some; b += some ? __builtin_ctzll(some) : 64) some = __ballot(b + lane >= a.n_seq || seq_of<R>(a, b + lane).nodes > 0);
      s = seq_of<R>(a, b);
    }
    const int pair = (u - first) / s.units, h = pair / s.tiles, tile = pair - h * s.tiles;
    const int t0 = u - first - pair * s.units, t1 = min(s.units, t0 + u_end - u);
    u += t1 - t0;
    const int32_t* table = a.table + (int64_t)b * a.n_table;
    const uint32_t* words[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int x = tile * R + nb * kCols + col, i = x / a.group, head = h * a.group + x - i * a.group;
      const bool there = i < s.nodes;
      t.node[nb] = there ? i : -1;
      words[nb] = a.mask + (int64_t)(s.first + (there ? i : 0)) * a.mask_words;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        t.q[nb][ks] = f16x8{};
        if (there) t.q[nb][ks] = *reinterpret_cast<const f16x8*>(a.q + ((int64_t)(s.first + i) * a.nq + head) * HD + ks * 32 + lg * 8);
      }
    }
    const int j_end = min(t1 * kUnit, s.keys);
    t.template blocks<false>(a, s, table, h, t0 * kUnit + w * kBlock, j_end, words, lane);
    if (!__all(t.finite())) t.template blocks<true>(a, s, table, h, t0 * kUnit + w * kBlock, j_end, words, lane);

    __syncthreads();                   // the pair before has been read
    if (lg == 0)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        s_ml[w][0][nb * kCols + col] = t.m[nb];
        s_ml[w][1][nb * kCols + col] = t.l[nb];
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
        for (int r = 0; r < 4; ++r) s_o[w][d][r][lane] = t.o[nb][d][r];
      __syncthreads();
      const int x = nb * kCols + c, i = (tile * R + x) / a.group, head = h * a.group + tile * R + x - i * a.group;
      if (i >= s.nodes) continue;
      float mx = -INFINITY, wt[kWaves], den = 0.f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) mx = fmaxf(mx, s_ml[v][0][x]);
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        const float mv = s_ml[v][0][x];
        wt[v] = mv == -INFINITY ? 0.f : exp2_hw(mv - mx);
        den += wt[v] * s_ml[v][1][x];
      }
      float acc[DPT];
#pragma unroll
      for (int e = 0; e < DPT; ++e) {
        const int dim = dbase + e;
        acc[e] = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) acc[e] += wt[v] * s_o[v][dim >> 4][dim & 3][((dim >> 2) & 3) * 16 + c];
      }
      if (t0 == 0 && t1 == s.units) {
        typedef _Float16 out_vec __attribute__((ext_vector_type(DPT)));
        const float inv = mx == -INFINITY ? 0.f : 1.0f / den;
        out_vec y;
#pragma unroll
        for (int e = 0; e < DPT; ++e) y[e] = (_Float16)(acc[e] * inv);
        *reinterpret_cast<out_vec*>(a.out + ((int64_t)(s.first + i) * a.nq + head) * HD + dbase) = y;
      } else {
        const int64_t e0 = (int64_t)(2 * g + (t0 == 0)) * R + x;
        if (dbase == 0) a.ml[e0] = make_float2(mx, den);
#pragma unroll
        for (int e = 0; e < DPT; e += 4)
          *reinterpret_cast<float4*>(a.part + e0 * HD + dbase + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
      }
    }
  }
}

// Joins the partials of one (row, query head): those of workgroups g0 .. g1.
// Group pg of LPP lanes takes partials pg, pg + NG, ... with their own running
// max, four dimensions a lane, and the groups meet in LDS; a partial's max, sum
// and values come in one trip to memory.
template <int HD, int R>
__global__ __launch_bounds__(256) void attn_tree_join_kernel(AttnTree a) {
  constexpr int LPP = HD / 4, NG = 256 / LPP, AHEAD = 4;     // lanes per partial, partials at once
  __shared__ float s_m[NG], s_l[NG];
  __shared__ f32x4 s_acc[NG][LPP];
  const int r = blockIdx.x / a.nq, hq = blockIdx.x % a.nq, h = hq / a.group;
  const int b = a.row_seq[r];
  if (b < 0) return;
  const Seq s = seq_of<R>(a, b);
  const int n_units = a.base[a.n_seq] * a.nkv, x = (r - s.first) * a.group + hq - h * a.group, tile = x / R, c = x - tile * R;
  const int t = threadIdx.x, dl = t % LPP, pg = t / LPP;
  const int nw = shares(a, n_units), f0 = a.base[b] * a.nkv + (h * s.tiles + tile) * s.units;
  const int g0 = share_of(f0, nw, n_units), n = share_of(f0 + s.units - 1, nw, n_units) - g0 + 1;
  if (n == 1) return;                              // written whole
  auto part = [&](int i) { return (int64_t)(2 * (g0 + i) + (i == 0)) * R + c; };
  float m = -INFINITY, l = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
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
      const float top = fmaxf(m, ml[k].x), old = m == top ? 1.f : exp2_hw(m - top), wt = exp2_hw(ml[k].x - top);
      m = top;
      l = l * old + wt * ml[k].y;
      acc = acc * old + v[k] * wt;
    }
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
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    const float inv = top == -INFINITY ? 0.f : 1.0f / den;
    *(reinterpret_cast<f16x4*>(a.out + (int64_t)blockIdx.x * HD) + dl) =
        f16x4{(_Float16)(acc[0] * inv), (_Float16)(acc[1] * inv), (_Float16)(acc[2] * inv), (_Float16)(acc[3] * inv)};
  }
}

int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

// Column blocks of a tile: as many as an average sequence fills, up to four.
int col_blocks(int64_t m, int n_seq, int group) {
  const int64_t cols = (m + n_seq - 1) / n_seq * group;
  return cols <= 16 ? 1 : cols <= 32 ? 2 : 4;
}

template <int HD, int NB>
void launch(const AttnTree& a, hipStream_t s) {
  const dim3 grid(a.wgs), block(64 * kWaves);
  if (a.C < kBlock)
    hipLaunchKernelGGL((attn_tree_kernel<HD, NB, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((attn_tree_kernel<HD, NB, false>), grid, block, 0, s, a);
  hipLaunchKernelGGL((attn_tree_join_kernel<HD, NB * kCols>), dim3(a.m * a.nq), dim3(256), 0, s, a);
}

template <int HD>
void launch(const AttnTree& a, int nb, hipStream_t s) {
  if (nb == 1) launch<HD, 1>(a, s);
  if (nb == 2) launch<HD, 2>(a, s);
  if (nb == 4) launch<HD, 4>(a, s);
}

}  // namespace

int64_t attention_tree_units(int m, int n_seq, int n_table, int chunk_tokens, int nq, int nkv) {
  const int64_t units = ((int64_t)n_table * chunk_tokens + kUnit - 1) / kUnit;
  const int64_t tiles = ((int64_t)m * (nq / nkv) + 15) / 16 + n_seq;
  return tiles * nkv * units;
}

int64_t attention_tree_ws_bytes(int m, int n_seq, int nq, int nkv, int hd) {
  // the partials of the widest tile, so that fewer rows, or more sequences, never need more
  const int64_t cols = (int64_t)2 * kWgs * 4 * kCols;
  return up256(((int64_t)n_seq + 1) * 4) + up256((int64_t)m * 4) + up256(cols * 8) + cols * hd * 4;
}

void launch_attention_tree(AttnTree a, int hd, void* ws, hipStream_t s) {
  uint8_t* p = reinterpret_cast<uint8_t*>(ws);
  const int nb = col_blocks(a.m, a.n_seq, a.group);
  a.base = reinterpret_cast<int32_t*>(p);
  p += up256(((int64_t)a.n_seq + 1) * 4);
  a.row_seq = reinterpret_cast<int32_t*>(p);
  p += up256((int64_t)a.m * 4);
  a.ml = reinterpret_cast<float2*>(p);
  p += up256((int64_t)2 * kWgs * nb * kCols * 8);
  a.part = reinterpret_cast<float*>(p);
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)hd);
  const int64_t most = attention_tree_units(a.m, a.n_seq, a.n_table, a.C, a.nq, a.nkv);
  a.wgs = most < kWgs ? (int)most : kWgs;
  if (hd == 128)
    launch<128>(a, nb, s);
  else
    launch<64>(a, nb, s);
}

}  // namespace mzk
