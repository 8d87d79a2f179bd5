// Appending the keys and values of many sequences to their chunked caches,
// rotated to their positions on the way, with the queries of the same rows
// rotated beside them (gfx950).
//
// Row r belongs to sequence seq[r] at position p = pos[r]; its chunk is
// table[seq][p / C], its place in the chunk p % C.  Keys and queries turn by
// the rotate-half pairs (i, i + hd/2) of rope.h; keys go token-major into the
// slot's K half, values dimension-major into its V^T half.  A row whose
// sequence or position lies outside the tables writes nothing, one whose
// chunk has no slot writes its query only.
//
// Memory-bound: every value is read once and written once.  Two kinds of
// workgroups in one launch: rotating ones, a thread per (four rows, run of
// pairs of one head), whose loads of the four rows are all in flight before
// the first is turned; and value ones, tiles of 64 rows x 64 dimensions
// turned through LDS, so that positions that follow each other leave as 16
// bytes per dimension and eight such runs as one line of V^T.  A decode row
// has no neighbour in its chunk: each of its values is a line of its own,
// which the slot layout asks for.
//
// Measured: 4099 f16 rows of 32 + 8 + 8 heads of 128 in 23.0 us, 103 MB at 4.5
// TB/s (a large copy: 4.6), with three inputs in turn; 18.6 with two, which the
// last-level cache partly holds.  64 fp32 rows one a sequence 6.0, 1 row 3.2 us,
// both latency.
#include "mz_kernels.h"
#include "rope.h"

namespace mzk {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr int kRotRows = 4;      // rows per thread of a rotating workgroup
constexpr int kValRows = 64;     // rows and dimensions of a value tile
constexpr int kValDims = 64;

// VEC consecutive values of a row as floats: 16 bytes of fp32 or f16.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  typedef float4 raw;
  static __device__ __forceinline__ void get(const raw& r, float (&v)[N]) {
    v[0] = r.x;
    v[1] = r.y;
    v[2] = r.z;
    v[3] = r.w;
  }
  typedef f16x4 half_vec;
};
template <>
struct Vec<_Float16> {
  static constexpr int N = 8;
  typedef f16x8 raw;
  static __device__ __forceinline__ void get(const raw& r, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)r[i];
  }
  typedef f16x8 half_vec;
};

// Whether row r's sequence and position lie inside the tables.
__device__ __forceinline__ bool row_ok(const KvAppend& a, int s, int p) {
  return (unsigned)s < (unsigned)a.n_seq && (unsigned)p < (unsigned)a.n_rope && (p >> a.cshift) < a.n_table;
}

template <typename T>
__device__ __forceinline__ void rotate_rows(const KvAppend& a, int m, int t, int items) {
  constexpr int N = Vec<T>::N;
  typedef typename Vec<T>::raw raw;
  const int halfd = a.hd / 2, per_head = halfd / N;
  const int rg = t / items, item = t - rg * items;
  const int head = item / per_head, i = (item - head * per_head) * N;
  const bool is_q = head < a.nq;
  const T* src = reinterpret_cast<const T*>(is_q ? a.q : a.k) + (is_q ? head : head - a.nq) * a.hd + i;
  const int64_t stride = is_q ? a.q_stride : a.k_stride;
  raw x1[kRotRows], x2[kRotRows];
  int s[kRotRows], p[kRotRows];
#pragma unroll
  for (int j = 0; j < kRotRows; ++j) {
    const int r = min(rg * kRotRows + j, m - 1);      // rows past the end repeat the last one's loads
    s[j] = a.seq[r];
    p[j] = a.pos[r];
    const T* x = src + (int64_t)r * stride;
    x1[j] = *reinterpret_cast<const raw*>(x);
    x2[j] = *reinterpret_cast<const raw*>(x + halfd);
  }
  int slot[kRotRows];
  float4 cs[kRotRows][N / 2];
#pragma unroll
  for (int j = 0; j < kRotRows; ++j) {
    const bool ok = row_ok(a, s[j], p[j]);
    slot[j] = ok ? 0 : -1;
    if (!is_q && ok) slot[j] = a.table[(int64_t)s[j] * a.n_table + (p[j] >> a.cshift)];
    const float4* c = reinterpret_cast<const float4*>(a.rope_cs + (int64_t)(ok ? p[j] : 0) * halfd + i);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) cs[j][e] = c[e];
  }
#pragma unroll
  for (int j = 0; j < kRotRows; ++j) {
    const int r = rg * kRotRows + j;
    if (r >= m || (unsigned)slot[j] >= (unsigned)a.n_slots) continue;
    float u[N], w[N];
    Vec<T>::get(x1[j], u);
    Vec<T>::get(x2[j], w);
    typename Vec<T>::half_vec y1, y2;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float4 c = cs[j][e / 2];
      const float2 y = rope_rotate(u[e], w[e], e & 1 ? c.z : c.x, e & 1 ? c.w : c.y);
      y1[e] = (_Float16)y.x;
      y2[e] = (_Float16)y.y;
    }
    _Float16* dst;
    if (is_q)
      dst = a.q_out + ((int64_t)r * a.nq + head) * a.hd + i;
    else
      dst = reinterpret_cast<_Float16*>(a.slab + (int64_t)slot[j] * a.slot_bytes) +
            ((int64_t)(p[j] & (a.C - 1)) * a.nkv + (head - a.nq)) * a.hd + i;
    *reinterpret_cast<typename Vec<T>::half_vec*>(dst) = y1;
    *reinterpret_cast<typename Vec<T>::half_vec*>(dst + halfd) = y2;
  }
}

// Value tile: rows r0 .. r0 + 63, dimensions d0 .. d0 + 63 of the dkv.  A run
// is eight rows that hold eight positions from a multiple of eight of one
// sequence (so one chunk: chunks hold a multiple of eight), wherever in the
// tile it begins; the rows outside runs leave value by value, lanes over
// rows, so that neighbours still meet in one line.
template <typename T>
__device__ __forceinline__ void value_tile(const KvAppend& a, int m, int r0, int d0, _Float16* tile, int64_t* s_at,
                                           int* s_run, int* s_one, int* s_n) {
  constexpr int N = Vec<T>::N, PITCH = kValDims + 2;
  typedef typename Vec<T>::raw raw;
  const int dkv = a.nkv * a.hd, dims = min(kValDims, dkv - d0), rows = min(kValRows, m - r0);
  constexpr int PER_ROW = kValDims / N, PER = kValRows * PER_ROW / 256;
  raw v[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int idx = threadIdx.x + 256 * e, r = min(idx / PER_ROW, rows - 1), d = (idx % PER_ROW) * N;
    v[e] = *reinterpret_cast<const raw*>(reinterpret_cast<const T*>(a.v) + (int64_t)(r0 + r) * a.v_stride + d0 +
                                         min(d, dims - N));
  }
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x, r = r0 + min(lane, rows - 1);
    const int s = a.seq[r], p = a.pos[r];
    int slot = -1;
    if (lane < rows && row_ok(a, s, p)) slot = a.table[(int64_t)s * a.n_table + (p >> a.cshift)];
    const bool ok = (unsigned)slot < (unsigned)a.n_slots;
    if (ok)
      s_at[lane] = (int64_t)slot * a.slot_bytes + (int64_t)a.C * dkv * 2 + (p & (a.C - 1)) * 2;
    const int s1 = __shfl_down(s, 1), p1 = __shfl_down(p, 1);
    const uint64_t okm = __ballot(ok);
    const uint64_t next = __ballot(ok && lane < 63 && s1 == s && p1 == p + 1) & (okm >> 1);
    const bool run = ok && (p & 7) == 0 && lane + 8 <= rows && ((next >> lane) & 0x7F) == 0x7F;
    const uint64_t runm = __ballot(run);
    uint64_t in_run = runm;
#pragma unroll
    for (int e = 1; e < 8; ++e) in_run |= runm << e;
    const uint64_t onem = okm & ~in_run, below = lane ? ~0ull >> (64 - lane) : 0ull;
    if (run) s_run[__popcll(runm & below)] = lane;
    if ((onem >> lane) & 1) s_one[__popcll(onem & below)] = lane;
    if (lane == 0) {
      s_n[0] = __popcll(runm);
      s_n[1] = __popcll(onem);
    }
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const int idx = threadIdx.x + 256 * e, r = idx / PER_ROW, d = (idx % PER_ROW) * N;
    float f[N];
    Vec<T>::get(v[e], f);
#pragma unroll
    for (int k = 0; k < N; ++k) tile[r * PITCH + d + k] = (_Float16)f[k];
  }
  __syncthreads();
  const int n_run = s_n[0], n_one = s_n[1];
  for (int idx = threadIdx.x; idx < n_run * dims; idx += 256) {
    const int d = idx / n_run, r = s_run[idx - d * n_run];
    f16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = tile[(r + e) * PITCH + d];
    *reinterpret_cast<f16x8*>(a.slab + s_at[r] + (int64_t)(d0 + d) * a.C * 2) = o;
  }
  for (int idx = threadIdx.x; idx < n_one * dims; idx += 256) {
    const int d = idx / n_one, r = s_one[idx - d * n_one];
    *reinterpret_cast<_Float16*>(a.slab + s_at[r] + (int64_t)(d0 + d) * a.C * 2) = tile[r * PITCH + d];
  }
}

template <typename T>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppend a, int m, int items, int rot_blocks) {
  __shared__ _Float16 tile[kValRows * (kValDims + 2)];
  __shared__ int64_t s_at[kValRows];
  __shared__ int s_run[8], s_one[kValRows], s_n[2];
  const int b = blockIdx.x;
  if (b < rot_blocks) {
    const int t = b * 256 + threadIdx.x;
    if (t < (m + kRotRows - 1) / kRotRows * items) rotate_rows<T>(a, m, t, items);
    return;
  }
  const int col_tiles = (a.nkv * a.hd + kValDims - 1) / kValDims, vb = b - rot_blocks;
  value_tile<T>(a, m, vb / col_tiles * kValRows, vb % col_tiles * kValDims, tile, s_at, s_run, s_one, s_n);
}

template <typename T>
int append_items(int nq, int nkv, int hd) {
  return (nq + nkv) * (hd / 2 / Vec<T>::N);
}

}  // namespace

bool kv_append_fits(int m, int nq, int nkv, int hd) {
  const int64_t groups = ((int64_t)m + kRotRows - 1) / kRotRows;
  const int64_t tiles = ((int64_t)m + kValRows - 1) / kValRows * ((nkv * hd + kValDims - 1) / kValDims);
  const int64_t threads = groups * append_items<float>(nq, nkv, hd);
  return threads < (int64_t(1) << 31) && threads / 256 + 1 + tiles <= kMaxBlocks;
}

void launch_kv_append(const KvAppend& a, int m, bool f32, hipStream_t s) {
  const int items = f32 ? append_items<float>(a.nq, a.nkv, a.hd) : append_items<_Float16>(a.nq, a.nkv, a.hd);
  const int rot = ((m + kRotRows - 1) / kRotRows * items + 255) / 256;
  const int tiles = (m + kValRows - 1) / kValRows * ((a.nkv * a.hd + kValDims - 1) / kValDims);
  if (f32)
    hipLaunchKernelGGL(kv_append_kernel<float>, dim3(rot + tiles), dim3(256), 0, s, a, m, items, rot);
  else
    hipLaunchKernelGGL(kv_append_kernel<_Float16>, dim3(rot + tiles), dim3(256), 0, s, a, m, items, rot);
}

}  // namespace mzk
