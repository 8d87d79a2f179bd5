// Rules on the logits of a batch of requests, and the token each row takes
// (gfx950).  For value x of token v in row i, with c occurrences of v in the
// row's history:
//   c > 0:  x = (x > 0 ? x / rep : x rep) - freq c - pres
//   v named by the row's biases:  x += the last of its entries
//   v's bit of the row's grammar mask is 0:  x = -inf
// then token = lowest index of the largest x, -1 where nothing is above -inf
// (NaN is never taken).  Each step is rounded to fp32 by itself.
//
// Memory-bound: the logits are read and written once.  A workgroup owns a
// slice of one row's vocabulary; it reads the row's whole history and bias
// list and keeps what falls into its slice in LDS, as counts (integer adds)
// and as the highest entry index per token (integer max), so neither needs
// vocabulary-sized memory, and the order in which lanes arrive changes
// nothing.  What a workgroup waits for is short and of one kind, so loads go
// out early (the first tokens of the history and the whole of a short bias
// list with the logits).  The slices' largest values meet in a second, small
// kernel.
//
// Measured (kernels, with penalties, biases, masks and tokens): 1 row of
// 128256, 2048 tokens held, 5.9 + 1.9 us, all latency; 64 rows of 151936, 4096
// tokens held, 25.2 us in all: 79 MB at 3.1 TB/s.  In a graph the same without
// lists 18.2, with one token held 21.1 (LDS is cleared and read), 2048 23.0,
// 4096 25.0, and with 300 biases 26.4.
#include "mz_kernels.h"

namespace mzk {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// (value, index) of the larger value, of the lower index where they are equal.
__device__ __forceinline__ void take(float& bv, int& bi, float ov, int oi) {
  if (ov > bv || (ov == bv && oi < bi)) {
    bv = ov;
    bi = oi;
  }
}

__device__ __forceinline__ void wave_best(float& bv, int& bi) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const float ov = __shfl_xor(bv, o);
    const int oi = __shfl_xor(bi, o);
    take(bv, bi, ov, oi);
  }
}

__device__ __forceinline__ float penalised(float x, float count, float rep, float freq, float pres) {
#pragma clang fp contract(off)
  const float held = x > 0.f ? x / rep : x * rep;
  const float f = count * freq;
  const float y = held - f;
  return y - pres;
}

// Threads and tokens of a workgroup.  1 row of 128256 (64), both kernels in a
// graph, with 100 biases: 7.9 (22.4) us; slices of 2048 7.3 (26.6), as every
// slice reads the row's lists; of 8192 9.2 (23.9).  256 threads: 9.4 (25.2).
constexpr int kThreads = 512, kSlice = 4096;

// History tokens and bias entries that the threads load ahead of the slice's
// other work, all together; what stands for a token without a bias: -0 as a
// value, below every index.
constexpr int kAheadHistory = 2048, kAheadBias = 512, kNone = (int)0x80000000;
constexpr int64_t kMostList = 1 << 30;      // entries of a row's list that are read

typedef int i32x4 __attribute__((ext_vector_type(4), aligned(4)));      // lists begin anywhere

// Tokens i .. i + 3 of a list, relative to v0; ~0 past its n entries.
__device__ __forceinline__ void tokens4(const int32_t* list, int i, int n, int v0, unsigned (&t)[4]) {
  if (i + 4 <= n) {
    const i32x4 u = *reinterpret_cast<const i32x4*>(list + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = (unsigned)u[e] - (unsigned)v0;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = i + e < n ? (unsigned)list[i + e] - (unsigned)v0 : ~0u;
  }
}

// VEC: logits a load, 4 where rows lie on 16-byte boundaries (22.3 us for 64
// rows of 128256, one by one 22.9).
template <int VEC>
__global__ __launch_bounds__(kThreads) void logits_rules_kernel(LogitsRules p) {
  constexpr int NT = kThreads, SLICE = kSlice, GROUPS = SLICE / (NT * VEC), AH = kAheadHistory / (4 * NT), AB = kAheadBias / NT;
  __shared__ __attribute__((aligned(16))) int s_count[SLICE];
  __shared__ __attribute__((aligned(16))) int s_last[SLICE];
  __shared__ float s_val[NT / 64];
  __shared__ int s_idx[NT / 64];
  const int row = blockIdx.x / p.slices, v0 = (blockIdx.x % p.slices) * SLICE, tid = threadIdx.x;
  const float* x = p.logits + (int64_t)row * p.stride;
  // value e of group i: token at(i) + e
  auto at = [&](int i) { return v0 + (i * NT + tid) * VEC; };
  float val[GROUPS][VEC];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int v = at(i);
    if (VEC == 4 && v + 4 <= p.vocab) {
      const f32x4 u = *reinterpret_cast<const f32x4*>(x + v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) val[i][e] = u[e & 3];
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) val[i][e] = v + e < p.vocab ? x[v + e] : -INFINITY;
    }
  }
  const int mask_row = !p.mask ? -1 : p.mask_row ? p.mask_row[row] : 0;
  uint32_t bits[GROUPS];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    bits[i] = ~0u;
    if ((unsigned)mask_row < (unsigned)p.n_masks && at(i) < p.vocab)
      bits[i] = p.mask[(int64_t)mask_row * p.mask_words + at(i) / 32] >> (at(i) & 31);
  }
  int64_t h0 = 0, h1 = p.n_history, b0 = 0, b1 = p.n_bias;
  if (p.history_off) h0 = p.history_off[row], h1 = p.history_off[row + 1];
  if (p.bias_off) b0 = p.bias_off[row], b1 = p.bias_off[row + 1];
  const int nh = (int)min(h1 - h0, kMostList), nb = (int)min(b1 - b0, kMostList);
  if (nh > 0 || nb > 0) {
    const unsigned here = (unsigned)min(SLICE, p.vocab - v0);
    const int32_t *history = p.history + h0, *bias_token = p.bias_token + b0;
    const float* bias_value = p.bias_value + b0;
    // tokens relative to the slice: inside it only below `here`
    unsigned ht[AH][4], bt[AB];
    float bval[AB];
    const bool held = nb <= NT * AB;       // the list's values stay in registers
#pragma unroll
    for (int k = 0; k < AH; ++k) tokens4(history, (tid + NT * k) * 4, nh, v0, ht[k]);
#pragma unroll
    for (int k = 0; k < AB; ++k) {
      const bool in = tid + NT * k < nb;
      bt[k] = in ? (unsigned)bias_token[tid + NT * k] - (unsigned)v0 : ~0u;
      bval[k] = in ? bias_value[tid + NT * k] : 0.f;
    }
    for (int i = tid * 4; i < SLICE; i += NT * 4) {
      *reinterpret_cast<int4*>(&s_count[i]) = make_int4(0, 0, 0, 0);
      *reinterpret_cast<int4*>(&s_last[i]) = make_int4(kNone, kNone, kNone, kNone);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < AH; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (ht[k][e] < here) atomicAdd(&s_count[ht[k][e]], 1);
#pragma unroll 2
    for (int i = (NT * AH + tid) * 4; i < nh; i += NT * 4) {
      unsigned t[4];
      tokens4(history, i, nh, v0, t);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (t[e] < here) atomicAdd(&s_count[t[e]], 1);
    }
    // entry e of the list stands as e + 1
#pragma unroll
    for (int k = 0; k < AB; ++k)
      if (bt[k] < here) atomicMax(&s_last[bt[k]], tid + NT * k + 1);
    for (int i = NT * AB + tid; i < nb; i += NT) {
      const unsigned t = (unsigned)bias_token[i] - (unsigned)v0;
      if (t < here) atomicMax(&s_last[t], i + 1);
    }
    __syncthreads();
    if (nb > 0 && held) {    // the last entry of a token puts its value in the place of its index
      bool last[AB];
#pragma unroll
      for (int k = 0; k < AB; ++k) last[k] = bt[k] < here && s_last[bt[k]] == tid + NT * k + 1;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < AB; ++k)
        if (last[k]) s_last[bt[k]] = __float_as_int(bval[k]);
      __syncthreads();
    }
    const float* pen = p.penalty + (int64_t)row * 3;
    const float rep = nh > 0 ? pen[0] : 1.f, freq = nh > 0 ? pen[1] : 0.f, pres = nh > 0 ? pen[2] : 0.f;
    // most waves hold no token of a list: what there is to do for one is left out whole
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      int c[VEC], last[VEC], any = 0, some = 0;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        c[e] = s_count[at(i) + e - v0];
        last[e] = s_last[at(i) + e - v0];
        any |= c[e];
        some |= last[e] != kNone;
      }
      if (__any(any)) {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (c[e] > 0) val[i][e] = penalised(val[i][e], (float)c[e], rep, freq, pres);
      }
      if (__any(some)) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          if (held)
            val[i][e] += __int_as_float(last[e]);      // -0 where there is no bias: it changes no value
          else if (last[e] != kNone)
            val[i][e] += bias_value[last[e] - 1];
        }
      }
    }
  }
  float bv = -INFINITY;
  int bi = 0x7fffffff;
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int v = at(i);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      if (!((bits[i] >> e) & 1)) val[i][e] = -INFINITY;
      if (val[i][e] > bv && v + e < p.vocab) {       // a thread's tokens ascend
        bv = val[i][e];
        bi = v + e;
      }
    }
    if (p.out) {
      float* o = p.out + (int64_t)row * p.stride + v;
      if (VEC == 4 && v + 4 <= p.vocab) {
        f32x4 u;
#pragma unroll
        for (int e = 0; e < VEC; ++e) u[e & 3] = val[i][e];
        *reinterpret_cast<f32x4*>(o) = u;
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (v + e < p.vocab) o[e] = val[i][e];
      }
    }
  }
  if (!p.token) return;
  wave_best(bv, bi);
  if ((tid & 63) == 0) {
    s_val[tid >> 6] = bv;
    s_idx[tid >> 6] = bi;
  }
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) take(bv, bi, s_val[i], s_idx[i]);
    p.part_val[blockIdx.x] = bv;
    p.part_idx[blockIdx.x] = bi;
  }
}

__global__ __launch_bounds__(64) void logits_token_kernel(LogitsRules p) {
  float bv = -INFINITY;
  int bi = 0x7fffffff;
  const int64_t first = (int64_t)blockIdx.x * p.slices;
  for (int i = threadIdx.x; i < p.slices; i += 64) take(bv, bi, p.part_val[first + i], p.part_idx[first + i]);
  wave_best(bv, bi);
  if (threadIdx.x == 0) p.token[blockIdx.x] = bi == 0x7fffffff ? -1 : bi;
}

int64_t slices_of(int vocab) { return ((int64_t)vocab + kSlice - 1) / kSlice; }

}  // namespace

// In 512-thread workgroups half of kMaxBlocks.
bool logits_rules_fits(int m, int vocab) { return slices_of(vocab) * m <= kMaxBlocks / 2; }

int64_t logits_rules_ws_bytes(int m, int vocab) { return slices_of(vocab) * m * 8; }

void launch_logits_rules(LogitsRules p, int m, void* ws, hipStream_t s) {
  p.slices = (int)slices_of(p.vocab);
  p.part_val = reinterpret_cast<float*>(ws);
  p.part_idx = reinterpret_cast<int32_t*>(p.part_val + (int64_t)m * p.slices);
  const bool vec = p.stride % 4 == 0 && ((uintptr_t)p.logits & 15) == 0 && ((uintptr_t)p.out & 15) == 0;
  const dim3 grid(m * p.slices);
  if (vec)
    hipLaunchKernelGGL(logits_rules_kernel<4>, grid, dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL(logits_rules_kernel<1>, grid, dim3(kThreads), 0, s, p);
  if (p.token) hipLaunchKernelGGL(logits_token_kernel, dim3(m), dim3(64), 0, s, p);
}

}  // namespace mzk
