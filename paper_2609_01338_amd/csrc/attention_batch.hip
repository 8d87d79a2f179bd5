// Attention of one new token of every sequence of a batch over its chunked KV
// cache (gfx950): for sequence b of len keys, head h of KV head h / G,
//   out = sum_j w_j v_j / sum_j w_j,  w_j = 2^(s_j - max s),
//   s_j = log2(e) / sqrt(hd) q . k_j,  j < len.
//
// Memory-bound: every key and value of the batch is read once (4 flops per query
// head for the 4 bytes of a key's and a value's dimension; a group of 4 heads is 4
// flops per byte).  So the work is cut by bytes, not by sequences: the units of
// 128 keys of all (sequence, KV head) pairs lie in one line, and each workgroup
// takes an even share of it, whatever the lengths, which are read here on the
// device.  A share that covers a pair whole writes its output; a pair that several
// shares meet leaves partials, at most two a workgroup (its first pair, begun by
// others, and its last, ended by others), and a second kernel joins them.
//
// A workgroup's four waves take the 32-key blocks of its share in turn.  The
// G query heads of the KV head are the 16-wide side of v_mfma_f32_16x16x32:
// S^T = K Q^T and O^T += V^T P^T with K and V^T fragments loaded straight
// from the slots, 16 bytes a lane: row i of the score product holds key
// 8 (i / 4) + 4 t + i % 4 of the block (t: first or second product), so that
// the eight scores of a lane are eight consecutive keys, and the P operand
// of the output product meets one 16-byte run of a V^T row.
//
// P goes into the product as two f16 values, hi + lo / 2^11, of 2^(14 + s - max),
// whose products are summed apart: 22 bits of a weight (and what they hold down
// to 2^-50 of the largest), so that nothing of an output's f16 is lost to the
// weights; matrix instructions are not what bounds this.  Their sum, the partials
// and the joins are fp32.
//
// Measured, both kernels, three inputs in turn: 64 sequences of 512-8192 keys, 8 KV
// heads of 128, 122 + 5 us: 640 MB at 5.2 TB/s, where only reading them in this
// order takes 117 us; one of 32768 28 + 5 (reading 31 with a workgroup a CU, as
// here, 29 with two); one of 2048, heads of 64, 5.4 + 4, latency.  With weights of
// one f16 the products took 0.2-0.8 us less.  Two and more blocks in flight a wave
// made the 64 sequences slower (137 us: the memory is busy, and what each share
// loads ahead in vain adds up); they were not tried with one workgroup a CU.
#include "mz_kernels.h"

namespace mzk {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kUnit = 128;          // keys of a unit: a 32-key block for each wave
constexpr int kWaves = 4, kBlock = 32, kCols = 16;
constexpr float kBias = 14.f;
constexpr float kLo = 2048.f;       // what a weight's lower half is multiplied by

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ int seq_len(const AttnBatch& a, int b) {
  return min(max(a.lens[b], 0), a.n_table << a.cshift);
}

// Workgroups that share `total` units.
__device__ __forceinline__ int shares(const AttnBatch& a, int total) { return min(a.wgs, total); }

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

template <int HD, bool SMALL>
__global__ __launch_bounds__(64 * kWaves, 2) void attn_batch_kernel(AttnBatch a) {
  constexpr int KS = HD / 32;          // 32-wide dimension steps of a score product
  constexpr int DB = HD / 16;          // 16-dimension blocks of the output
  __shared__ float s_o[kWaves][DB][4][64];
  __shared__ float s_ml[kWaves][2][kCols];
  __shared__ int s_red[kWaves], s_at[2];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, lg = lane >> 4;
  const int dkv = a.nkv * HD;

  // where this workgroup's share begins: (sequence, units of the sequences before it)
  int total = 0, u_mine = 0, u_before = 0;
  for (int b0 = 0; b0 < a.n_seq; b0 += 256) {
    const int b = b0 + threadIdx.x;
    u_mine = b < a.n_seq ? (seq_len(a, b) + kUnit - 1) / kUnit : 0;
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
      u_mine = b < a.n_seq ? (seq_len(a, b) + kUnit - 1) / kUnit : 0;
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

  int len = seq_len(a, b);
  while (u < u_end) {
    int nu = (len + kUnit - 1) / kUnit;
    if (u >= first + nu * a.nkv) {       // past this sequence: on to the next that has keys, 64 in a look
      first += nu * a.nkv;
      uint64_t some = 0;
      for (++b; !some; b += some ? __builtin_ctzll(some) : 64) {
        len = b + lane < a.n_seq ? seq_len(a, b + lane) : 1;
        some = __ballot(len > 0);
      }
      len = __builtin_amdgcn_readlane(len, __builtin_ctzll(some));
      nu = (len + kUnit - 1) / kUnit;
    }
    const int h = (u - first) / nu, t0 = u - first - h * nu, t1 = min(nu, t0 + u_end - u);
    u += t1 - t0;
    const int32_t* table = a.table + (int64_t)b * a.n_table;
    f16x8 bq[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      bq[ks] = f16x8{};
      if (col < a.group)
        bq[ks] = *reinterpret_cast<const f16x8*>(a.q + ((int64_t)b * a.nq + h * a.group + col) * HD + ks * 32 + lg * 8);
    }
    f32x4 o[DB], o_lo[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = o_lo[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_c = -INFINITY, l_c = 0.f;

    // This wave's blocks: j0, j0 + 128, ... below the share's end and the
    // sequence's.  Table entries are read a block ahead, so that a block waits
    // for one trip to memory, not two.
    const int j_end = min(t1 * kUnit, len), last = len - 1;
    Slots next = slots_of<SMALL>(table, a.cshift, min(t0 * kUnit + w * kBlock, last), col, lg, last);
    for (int j0 = t0 * kUnit + w * kBlock; j0 < j_end; j0 += kUnit) {
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

      f32x4 sc[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ka[t][ks], bq[ks], sc[t], 0, 0, 0);
      }
      // A key that counts raises the running max to at least the lowest fp32
      // value, so -inf means that none was seen; scores of -inf and NaN then
      // go where the formula sends them.
      const int n_ok = ok ? len - vj : 0;     // keys vj .. vj + n_ok - 1 of this lane's eight count
      float bm = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool in = 4 * t + r < n_ok;
          const float v = sc[t][r] * a.scale_log2;
          sc[t][r] = in ? v : -INFINITY;
          bm = in ? fmaxf(bm, fmaxf(v, -3.402823466e38f)) : bm;
        }
      bm = fmaxf(bm, __shfl_xor(bm, 16));
      bm = fmaxf(bm, __shfl_xor(bm, 32));
      if (__any(bm > m_c)) {
        const float m_new = fmaxf(m_c, bm);
        const float alpha = m_new == m_c ? 1.f : exp2_hw(m_c - m_new);
        m_c = m_new;
        l_c *= alpha;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] *= alpha, o_lo[d] *= alpha;
      }
      const float base = m_c == -INFINITY ? 0.f : m_c - kBias;
      f16x8 pb, pb_lo;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float e = exp2_hw(sc[t][r] - base);
          const _Float16 hi = (_Float16)e;
          pb[t * 4 + r] = hi;
          pb_lo[t * 4 + r] = (_Float16)((e - (float)hi) * kLo);
          l_c += e;
        }
      // values of keys that do not count are not data: zero them
      if (__any(n_ok < 8)) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e = 0; e < 8; ++e) va[d][e] = e < n_ok ? va[d][e] : (_Float16)0.f;
      }
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va[d], pb, o[d], 0, 0, 0);
        o_lo[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va[d], pb_lo, o_lo[d], 0, 0, 0);
      }
    }
    l_c += __shfl_xor(l_c, 16);
    l_c += __shfl_xor(l_c, 32);
    __syncthreads();                   // the pair before has been read
    if (lg == 0) {
      s_ml[w][0][col] = m_c;
      s_ml[w][1][col] = l_c;
    }
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r)      // a sum with infinite or NaN values is what the upper halves make of it
        s_o[w][d][r][lane] = fabsf(o[d][r]) < INFINITY ? __builtin_fmaf(o_lo[d][r], 1.f / kLo, o[d][r]) : o[d][r];
    __syncthreads();
    // thread t: head t % 16 of the group, output dimensions (t / 16) * DPT .. + DPT
    constexpr int DPT = HD / 16;
    const int c = threadIdx.x & 15, dbase = (threadIdx.x >> 4) * DPT;
    if (c < a.group) {
      float mx = -INFINITY, wt[kWaves], den = 0.f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) mx = fmaxf(mx, s_ml[v][0][c]);
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        const float mv = s_ml[v][0][c];
        wt[v] = mv == -INFINITY ? 0.f : exp2_hw(mv - mx);
        den += wt[v] * s_ml[v][1][c];
      }
      float acc[DPT];
#pragma unroll
      for (int e = 0; e < DPT; ++e) {
        const int dim = dbase + e;
        acc[e] = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) acc[e] += wt[v] * s_o[v][dim >> 4][dim & 3][((dim >> 2) & 3) * 16 + c];
      }
      if (t0 == 0 && t1 == nu) {
        typedef _Float16 out_vec __attribute__((ext_vector_type(DPT)));
        const float inv = mx == -INFINITY ? 0.f : 1.0f / den;
        out_vec y;
#pragma unroll
        for (int e = 0; e < DPT; ++e) y[e] = (_Float16)(acc[e] * inv);
        *reinterpret_cast<out_vec*>(a.out + ((int64_t)b * a.nq + h * a.group + c) * HD + dbase) = y;
      } else {
        const int64_t e0 = (int64_t)(2 * g + (t0 == 0)) * a.group + c;
        if (dbase == 0) a.ml[e0] = make_float2(mx, den);
#pragma unroll
        for (int e = 0; e < DPT; e += 4)
          *reinterpret_cast<float4*>(a.part + e0 * HD + dbase + e) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
      }
    }
  }
}

// Joins the partials of one (sequence, query head): those of workgroups g0 ..
// g1.  Group pg of LPP lanes takes partials pg, pg + NG, ... with their own
// running max, four dimensions a lane, and the groups meet in LDS; a partial's
// max, sum and values come in one trip to memory.
template <int HD>
__global__ __launch_bounds__(256) void attn_batch_join_kernel(AttnBatch a) {
  constexpr int LPP = HD / 4, NG = 256 / LPP, AHEAD = 4;     // lanes per partial, partials at once
  __shared__ float s_m[NG], s_l[NG];
  __shared__ f32x4 s_acc[NG][LPP];
  const int b = blockIdx.x / a.nq, hq = blockIdx.x % a.nq, h = hq / a.group, c = hq % a.group;
  const int u0 = a.base[b], nu = a.base[b + 1] - u0, n_units = a.base[a.n_seq] * a.nkv;
  const int t = threadIdx.x, dl = t % LPP, pg = t / LPP;
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  f16x4* out = reinterpret_cast<f16x4*>(a.out + (int64_t)blockIdx.x * HD) + dl;
  if (nu == 0) {
    if (pg == 0) *out = f16x4{0, 0, 0, 0};
    return;
  }
  const int nw = shares(a, n_units), f0 = u0 * a.nkv + h * nu;
  const int g0 = share_of(f0, nw, n_units), n = share_of(f0 + nu - 1, nw, n_units) - g0 + 1;
  if (n == 1) return;                              // written whole
  auto part = [&](int i) { return (int64_t)(2 * (g0 + i) + (i == 0)) * a.group + c; };
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
    const float inv = top == -INFINITY ? 0.f : 1.0f / den;
    *out = f16x4{(_Float16)(acc[0] * inv), (_Float16)(acc[1] * inv), (_Float16)(acc[2] * inv), (_Float16)(acc[3] * inv)};
  }
}

// Shares: one workgroup a CU where pairs are few (a share's keys are then
// mostly one pair's, and fewer partials are joined), two where they are many
// (what a pair costs beside its keys, its queries, its table and the waves'
// join, hides behind the other workgroup).  256 against 512 (768) shares,
// both kernels in a graph, 4 query heads a KV head, dimension 128: 8 pairs of
// 12000 keys 16.5 against 18.5 (17.9) us, of 32768 28.2 against 28.9 (29.4);
// 128 pairs of 260-4096 26.7 against 28.1 (26.1), 200 of 1000 25.8 against 27.2
// (26.5); 256 pairs of 1000 26.2 against 28.1 (28.2), of 260-4096 40.8 against
// 37.3 (37.4), so the border lies where lengths decide; 320 pairs of 1000 33.1
// against 33.4 (34.0), of 260-4096 51.1 against 45.5 (45.3); 512 pairs of 50
// 11.8 against 10.3 (10.2), of 300 22.5 against 20.6 (23.7), of 1000 47.0 against
// 46.6 (49.8); dimension 64, 512 pairs of 130-2048 31.6 against 25.2 (24.4), of
// 1000 28.6 against 27.2 (30.7).
constexpr int kFewPairs = 256;

int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

}  // namespace

int64_t attention_batch_units(int n_seq, int n_table, int chunk_tokens, int n_kv) {
  return ((int64_t)n_table * chunk_tokens + kUnit - 1) / kUnit * n_seq * n_kv;
}

int64_t attention_batch_ws_bytes(int n_seq, int group, int hd) {
  return up256(((int64_t)n_seq + 1) * 4) + up256((int64_t)2 * kAttnBatchWgs * group * 8) +
         (int64_t)2 * kAttnBatchWgs * group * hd * 4;
}

void launch_attention_batch(AttnBatch a, int hd, void* ws, hipStream_t s) {
  uint8_t* p = reinterpret_cast<uint8_t*>(ws);
  a.base = reinterpret_cast<int32_t*>(p);
  a.ml = reinterpret_cast<float2*>(p + up256(((int64_t)a.n_seq + 1) * 4));
  a.part = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(a.ml) + up256((int64_t)2 * kAttnBatchWgs * a.group * 8));
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)hd);
  const int64_t most = attention_batch_units(a.n_seq, a.n_table, a.C, a.nkv);
  a.wgs = (int64_t)a.n_seq * a.nkv <= kFewPairs ? kAttnBatchWgs / 2 : kAttnBatchWgs;
  if (most < a.wgs) a.wgs = (int)most;
  const dim3 grid(a.wgs), block(64 * kWaves);
  if (hd == 128) {
    if (a.C < kBlock)
      hipLaunchKernelGGL((attn_batch_kernel<128, true>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((attn_batch_kernel<128, false>), grid, block, 0, s, a);
    hipLaunchKernelGGL(attn_batch_join_kernel<128>, dim3(a.n_seq * a.nq), dim3(256), 0, s, a);
  } else {
    if (a.C < kBlock)
      hipLaunchKernelGGL((attn_batch_kernel<64, true>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((attn_batch_kernel<64, false>), grid, block, 0, s, a);
    hipLaunchKernelGGL(attn_batch_join_kernel<64>, dim3(a.n_seq * a.nq), dim3(256), 0, s, a);
  }
}

}  // namespace mzk
