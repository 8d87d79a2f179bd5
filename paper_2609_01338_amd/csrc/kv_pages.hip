// Which slots of the slab the sequences hold from now on, and the copies that
// this asks for (gfx950).
//
// new[b][c] = old[src_b][c] for the chunks of the first keep_b keys, and fresh
// slots behind them up to keep + room.  No count of a slot's holders outlives
// the call: they are counted from the kept entries (integer additions, whose
// order does not matter), and a slot that nobody keeps is free.  A row that
// writes into a chunk kept in part takes a copy if others hold it; if all of them
// write, the one with the lowest order (rows that stay first) keeps it.  Wanted
// slots (for slots past the limit, ascending; then row by row) and free slots
// are numbered by prefix sums, and the k-th wanted one gets the k-th free one.
#include "mz_kernels.h"

namespace mzk {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

enum { kSumMoves, kSumMissing };       // in KvPages::sums

struct Span {
  int src, keep, end, edge;      // edge: the chunk that holds position keep
  bool partial;                  // it holds kept keys and is written
};
__device__ __forceinline__ Span span_of(const KvPages& a, int b) {
  Span s;
  const int top = a.n_table << a.cshift;
  s.src = a.src ? a.src[b] : b;
  s.keep = (unsigned)s.src < (unsigned)a.n_seq ? min(max(a.keep[b], 0), top) : 0;
  const int room = a.room ? max(a.room[b], 0) : 0;
  s.end = room < top - s.keep ? s.keep + room : top;
  s.edge = s.keep >> a.cshift;
  s.partial = s.end > s.keep && (s.keep & (a.C - 1)) != 0;
  return s;
}

// What rows take a copy of slot e: all that write it, but one if nobody else holds it.
__device__ __forceinline__ int copies_of(int count, int writers) {
  return count <= 1 ? 0 : writers == count ? count - 1 : writers;
}

__global__ __launch_bounds__(256) void pages_clear_kernel(KvPages a) {
  const int s = blockIdx.x * 256 + threadIdx.x;
  if (s >= a.n_slots) return;
  a.count[s] = a.writers[s] = 0;
  a.lowest[s] = 2 * a.n_seq;
}

__global__ __launch_bounds__(256) void pages_kept_kernel(KvPages a) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (int64_t)a.n_seq * a.n_table) return;
  const int b = (int)(at / a.n_table), c = (int)(at - (int64_t)b * a.n_table);
  const Span s = span_of(a, b);
  int e = -1;
  if (c <= (s.keep - 1) >> a.cshift) e = a.table[(int64_t)s.src * a.n_table + c];
  if ((unsigned)e >= (unsigned)a.n_slots) e = -1;
  a.kept[at] = e;
  if (e < 0) return;
  atomicAdd(&a.count[e], 1);
  if (s.partial && c == s.edge) {
    atomicAdd(&a.writers[e], 1);
    atomicMin(&a.lowest[e], s.src == b ? b : a.n_seq + b);
  }
}

// Inclusive sums over the 1024 threads; sum: of all.
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
  for (int i = 0; i < 16; ++i) {
    if (i < w) before += red[i];
    sum += red[i];
  }
  return v + before;
}

constexpr int kPer = 8;        // slots of a thread at once

__global__ __launch_bounds__(1024) void pages_number_kernel(KvPages a) {
  __shared__ int red[16];
  int n_free = 0, n_moves = 0, n_held = 0;
  for (int s0 = 0; s0 < a.n_slots; s0 += 1024 * kPer) {
    const int first = s0 + threadIdx.x * kPer;
    int count[kPer], writers[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int s = min(first + e, a.n_slots - 1);
      count[e] = a.count[s];
      writers[e] = s >= a.limit ? a.writers[s] : 0;
    }
    int free = 0, moves = 0, held = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int s = first + e;
      free += s < a.limit && count[e] == 0;
      moves += s >= a.limit && s < a.n_slots && count[e] > copies_of(count[e], writers[e]);
      held += s < a.n_slots && count[e] > 0;
    }
    int sum;
    int f = n_free + block_scan(free, red, sum) - free;
    n_free += sum;
    int mv = n_moves + block_scan(moves, red, sum) - moves;
    n_moves += sum;
    block_scan(held, red, sum);
    n_held += sum;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int s = first + e;
      if (s < a.limit && count[e] == 0) a.free_at[f++] = s;
      if (s >= a.limit && s < a.n_slots) a.moved_to[s] = count[e] > copies_of(count[e], writers[e]) ? mv++ : -1;
    }
  }
  int64_t wanted = n_moves;
  int n_forks = 0;
  for (int b0 = 0; b0 < a.n_seq; b0 += 1024) {
    const int b = b0 + threadIdx.x;
    int need = 0, fork = 0;
    if (b < a.n_seq) {
      const Span s = span_of(a, b);
      if (s.end > s.keep) {
        need = ((s.end - 1) >> a.cshift) - s.edge + 1;
        const int e = s.partial ? a.kept[(int64_t)b * a.n_table + s.edge] : -1;
        if (e >= 0) {
          const int count = a.count[e];
          const bool stays = count == 1 || (a.writers[e] == count && a.lowest[e] == (s.src == b ? b : a.n_seq + b));
          fork = !stays;
          need -= stays;
        }
      }
    }
    int sum;
    const int before = block_scan(need, red, sum) - need;
    const int64_t at = wanted + before;
    wanted += sum;
    const int f = n_forks + block_scan(fork, red, sum) - fork;
    n_forks += sum;
    if (b < a.n_seq) {
      a.need[b] = (int)(at < INT32_MAX ? at : INT32_MAX);
      a.forks[b] = fork ? f : -1;
    }
  }
  if (threadIdx.x == 0) {
    const int missing = wanted > n_free ? (int)(wanted - n_free) : 0;
    a.sums[kSumMoves] = n_moves;
    a.sums[kSumMissing] = missing;
    a.info[0] = missing;
    a.info[1] = (int)(n_held + wanted - n_moves);
    a.info[2] = missing ? 0 : n_moves + n_forks;
    a.info[3] = 0;
  }
}

__global__ __launch_bounds__(256) void pages_take_kernel(KvPages a) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const bool missing = a.sums[kSumMissing] > 0;
  const int n_moves = a.sums[kSumMoves];
  if (!missing && at >= a.limit && at < a.n_slots) {
    const int k = a.moved_to[at];
    if (k >= 0) a.copies[k] = make_int4((int)at, a.free_at[k], a.C, 0);
  }
  if (at >= (int64_t)a.n_seq * a.n_table) return;
  if (missing) {
    a.table_out[at] = a.table[at];
    return;
  }
  const int b = (int)(at / a.n_table), c = (int)(at - (int64_t)b * a.n_table);
  const Span s = span_of(a, b);
  int e = a.kept[at];
  const bool written = s.end > s.keep && c >= s.edge && c <= (s.end - 1) >> a.cshift;
  if (written) {
    const int edge = s.partial ? (c == s.edge ? e : a.kept[(int64_t)b * a.n_table + s.edge]) : -1;
    const int fork = a.forks[b];
    if (c == s.edge && edge >= 0 && fork >= 0) {
      const int to = a.free_at[a.need[b]];
      a.copies[n_moves + fork] = make_int4(e, to, s.keep & (a.C - 1), 0);
      a.table_out[at] = to;
      return;
    }
    if (c > s.edge || edge < 0) {
      a.table_out[at] = a.free_at[a.need[b] + c - s.edge - (edge >= 0 && fork < 0)];
      return;
    }
  }
  a.table_out[at] = e >= a.limit ? a.free_at[a.moved_to[e]] : e;
}

// A workgroup takes pieces of 256 x 8 times 16 bytes of a (copy, layer): first
// of the key rows, then of the V^T rows, of which a run of 8 positions that
// holds the last one is written value by value.
constexpr int kPiece = 8;

__global__ __launch_bounds__(256) void kv_copy_kernel(KvCopy a, int pieces) {
  const int n = min(max(*a.n_copies, 0), a.max_copies);
  const int64_t items = (int64_t)n * a.n_layers * pieces;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t at = item / pieces;
    const int piece = (int)(item - at * pieces);
    const int layer = (int)(at / n), i = (int)(at - (int64_t)layer * n);
    const int4 c = a.copies[i];
    if ((unsigned)c.x >= (unsigned)a.n_slots || (unsigned)c.y >= (unsigned)a.n_slots || c.x == c.y) continue;
    const int tokens = min(max(c.z, 0), a.C), runs = (tokens + 7) / 8, keys = tokens * (a.dkv / 8);
    const int units = keys + a.dkv * runs;
    const uint8_t* from = a.slab + layer * a.layer_bytes + c.x * a.slot_bytes;
    uint8_t* to = a.slab + layer * a.layer_bytes + c.y * a.slot_bytes;
    f16x8 x[kPiece];
    unsigned off[kPiece];
    int last[kPiece];            // values of the unit that count
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
      const int u = (piece * kPiece + e) * 256 + threadIdx.x;
      last[e] = 0;
      if (u < units) {
        const int v = u - keys, d = v < 0 ? 0 : v / runs, run = v - d * runs;
        off[e] = v < 0 ? (unsigned)u * 16u : ((unsigned)a.dkv + d) * (unsigned)a.C * 2u + run * 16u;
        last[e] = v < 0 ? 8 : min(8, tokens - run * 8);
        x[e] = *reinterpret_cast<const f16x8*>(from + off[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
      if (last[e] == 8)
        *reinterpret_cast<f16x8*>(to + off[e]) = x[e];
      else
#pragma unroll
        for (int j = 0; j < 7; ++j)
          if (j < last[e]) *reinterpret_cast<_Float16*>(to + off[e] + j * 2) = x[e][j];
    }
  }
}

int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

}  // namespace

int64_t kv_pages_ws_bytes(int n_seq, int n_table, int n_slots) {
  return up256((int64_t)n_seq * n_table * 4) + 5 * up256((int64_t)n_slots * 4) + 2 * up256((int64_t)n_seq * 4) + 256;
}

void launch_kv_pages(KvPages a, void* ws, hipStream_t s) {
  uint8_t* p = reinterpret_cast<uint8_t*>(ws);
  auto take = [&](int64_t n) {
    int32_t* at = reinterpret_cast<int32_t*>(p);
    p += up256(n * 4);
    return at;
  };
  const int64_t entries = (int64_t)a.n_seq * a.n_table;
  a.kept = take(entries);
  a.count = take(a.n_slots);
  a.writers = take(a.n_slots);
  a.lowest = take(a.n_slots);
  a.free_at = take(a.n_slots);
  a.moved_to = take(a.n_slots);
  a.need = take(a.n_seq);
  a.forks = take(a.n_seq);
  a.sums = take(8);
  const int64_t both = entries > a.n_slots ? entries : a.n_slots;
  hipLaunchKernelGGL(pages_clear_kernel, dim3((a.n_slots + 255) / 256), dim3(256), 0, s, a);
  hipLaunchKernelGGL(pages_kept_kernel, dim3((unsigned)((entries + 255) / 256)), dim3(256), 0, s, a);
  hipLaunchKernelGGL(pages_number_kernel, dim3(1), dim3(1024), 0, s, a);
  hipLaunchKernelGGL(pages_take_kernel, dim3((unsigned)((both + 255) / 256)), dim3(256), 0, s, a);
}

void launch_kv_copy(const KvCopy& a, hipStream_t s) {
  const int64_t units = a.slot_bytes / 16;
  const int pieces = (int)((units + 256 * kPiece - 1) / (256 * kPiece));
  const int64_t items = (int64_t)a.max_copies * a.n_layers * pieces;
  hipLaunchKernelGGL(kv_copy_kernel, dim3((unsigned)(items < 2048 ? items : 2048)), dim3(256), 0, s, a, pieces);
}

}  // namespace mzk
