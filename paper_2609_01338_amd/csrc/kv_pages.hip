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
//
// All of it is latency: a table of 64 rows of 257 entries over 7000 slots is 66 KB.
// Up to kSmallSlots slots, kSmallRows rows and kSmallEntries entries one workgroup
// does it with the counts in LDS (16 bits of holders and 16 of writers a slot), else four
// launches do.
//
// The copies are a launch of their own: 16 KB pieces, a workgroup each up to 8192 of
// them, stored past the caches.  Of 16 layers of 1 MB slots, 50 moves and 12
// forks, it takes 118 us at 4.8 TB/s (a large copy: 4.6; 2048 workgroups of 32 KB
// pieces in turn, stored through the caches, 156).
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

// Inclusive sums over the 1024 threads; sum: of all.  v holds several numbers in bits of their own.
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t* red, uint64_t& sum) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();
  if (lane == 63) red[w] = v;
  __syncthreads();
  uint64_t before = 0;
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
  __shared__ uint64_t red[16];
  constexpr int BITS = 20;             // of the counts of 1024 kPer slots: free, moves, held
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
    uint64_t mine = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int s = first + e;
      mine += (uint64_t)(s < a.limit && count[e] == 0);
      mine += (uint64_t)(s >= a.limit && s < a.n_slots && count[e] > copies_of(count[e], writers[e])) << BITS;
      mine += (uint64_t)(s < a.n_slots && count[e] > 0) << 2 * BITS;
    }
    uint64_t sum;
    const uint64_t before = block_scan(mine, red, sum) - mine;
    int f = n_free + (int)(before & ((1 << BITS) - 1)), mv = n_moves + (int)(before >> BITS & ((1 << BITS) - 1));
    n_free += (int)(sum & ((1 << BITS) - 1));
    n_moves += (int)(sum >> BITS & ((1 << BITS) - 1));
    n_held += (int)(sum >> 2 * BITS);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int s = first + e;
      if (s < a.limit && count[e] == 0) a.free_at[f++] = s;
      if (s >= a.limit && s < a.n_slots) a.moved_to[s] = count[e] > copies_of(count[e], writers[e]) ? mv++ : -1;
    }
  }
  int64_t wanted = n_moves;            // at most 2^28 of each kind
  int n_forks = 0;
  for (int b0 = 0; b0 < a.n_seq; b0 += 1024) {
    const int b = b0 + threadIdx.x;
    int need = 0;
    bool fork = false;
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
    const uint64_t mine = (uint64_t)need | (uint64_t)fork << 40;
    uint64_t sum;
    const uint64_t before = block_scan(mine, red, sum) - mine;
    const int64_t at = wanted + (int64_t)(before & ((1ull << 40) - 1));
    if (b < a.n_seq) {
      a.need[b] = (int)(at < INT32_MAX ? at : INT32_MAX);
      a.forks[b] = fork ? n_forks + (int)(before >> 40) : -1;
    }
    wanted += (int64_t)(sum & ((1ull << 40) - 1));
    n_forks += (int)(sum >> 40);
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

// ---- all of it in one workgroup
// It takes its entries in turns of 8192, with two trips to memory in each, where four
// launches have a start of their own.  us of one workgroup / four launches, in a graph and, in
// brackets, called alone and waited for:
//   entries      16 rows, 8192 slots          64 rows, 8192 slots        320 rows, 8192   1024, 3000
//      8192   11.9 / 15.5                  11.9 / 15.9                                    10.6 / 25.9
//     16384   15.4 / 15.9 (30.5 / 32.9)    15.6 / 16.0 (30.5 / 33.8)                      14.3 / 26.2
//     20480   18.4 / 16.4 (33.3 / 33.6)    18.5 / 16.6 (33.3 / 33.7)    19.1 / 19.8       17.3 / 25.9
//     24576                                19.1 / 17.1 (34.1 / 34.1)
//     32768                                22.7 / 17.0 (37.4 / 34.0)
// Among a step's other launches from Python 64 rows of 257 entries over 7000 slots are 16.8 /
// 21.5 with the empty copy behind them, 17.5 / 16.9 in a graph.  The limit is the number at which few rows
// called alone take as long either way, in a graph 2 us too high for few rows and
// too low for many.  (Where all of many rows write the one chunk that they share, each looks
// at the others: 1024 rows 69 / 25.)
constexpr int kSmallSlots = 8192, kSmallRows = 1024, kSmallEntries = 20480;

// Which threads of the wave below this one have `on`, and how many have it in all.
__device__ __forceinline__ int rank_of(uint64_t on) {
  const int lane = threadIdx.x & 63;
  return __popcll(on & (lane ? ~0ull >> (64 - lane) : 0));
}

__global__ __launch_bounds__(1024) void pages_small_kernel(KvPages a) {
  __shared__ unsigned s_slot[kSmallSlots];                   // holders, writers << 16; then the number of a slot that moves
  __shared__ int4 s_row[kSmallRows];                   // first the source's entries, chunks kept, the one kept in part and written;
                                                       // then first and last chunk written, number of the wanted slot less the
                                                       // chunk, number of the first chunk's (-1: none)
  __shared__ int s_src[kSmallRows], s_edge[kSmallRows], s_fork[kSmallRows];
  __shared__ int s_sum[16][5];                         // of a wave: free, moves, held; wanted, forks
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int entries = a.n_seq * a.n_table;
  for (int s = t; s < a.n_slots; s += 1024) s_slot[s] = 0;
  Span mine{};
  if (t < a.n_seq) {
    mine = span_of(a, t);
    s_row[t] = make_int4(mine.keep ? mine.src * a.n_table : 0, (mine.keep + a.C - 1) >> a.cshift, mine.partial ? mine.edge : -1, 0);
    s_src[t] = mine.src;
    s_edge[t] = -1;
  }
  __syncthreads();
  // the entries that are kept, eight of a thread in one trip to memory
  constexpr int PER = 8;
  // (i + 0.5) / n_table lies at least 0.5 / n_table from a whole number, and for i below 2^16
  // the two roundings are a hundredth of that)
  const float per_row = 1.f / (float)a.n_table;
  auto row_of = [&](int i) { return (int)(((float)i + 0.5f) * per_row); };
  for (int i0 = t; i0 < entries; i0 += 1024 * PER) {
    int e[PER], edge[PER];             // edge: the row, where the entry is of the chunk kept in part and written, else -1
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = min(i0 + 1024 * k, entries - 1), b = row_of(i), c = i - b * a.n_table;
      const int4 row = s_row[b];
      e[k] = c < row.y ? a.table[row.x + c] : -1;
      edge[k] = c == row.z ? b : -1;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = i0 + 1024 * k;
      if (i >= entries) break;
      if ((unsigned)e[k] >= (unsigned)a.n_slots) e[k] = -1;
      a.kept[i] = e[k];
      if (e[k] < 0) continue;
      if (edge[k] >= 0) s_edge[edge[k]] = e[k];
      atomicAdd(&s_slot[e[k]], edge[k] >= 0 ? 0x10001u : 1u);
    }
  }
  __syncthreads();
  // rows: what they want, and whether they take a copy
  int need = 0;
  bool fork = false;
  if (mine.end > mine.keep) {
    const int edge = s_edge[t];
    need = ((mine.end - 1) >> a.cshift) - mine.edge + 1;
    if (edge >= 0) {
      const unsigned x = s_slot[edge];
      const int holders = x & 0xFFFF, writers = x >> 16;
      fork = holders > 1;
      if (holders > 1 && holders == writers) {
        const int order = mine.src == t ? t : a.n_seq + t;
        fork = false;
        for (int b = 0; b < a.n_seq; ++b) fork |= s_edge[b] == edge && (s_src[b] == b ? b : a.n_seq + b) < order;
      }
      need -= !fork;
    }
  }
  // slots: each wave numbers those of its part of them
  const int part = ((a.n_slots + 15) / 16 + 63) / 64 * 64, s0 = w * part, s1 = min(s0 + part, a.n_slots);
  auto look = [&](int s, bool& free, bool& moves, bool& held) {
    const unsigned x = s < s1 ? s_slot[s] : 0;
    held = (x & 0xFFFF) > 0;
    free = s < s1 && s < a.limit && !held;
    moves = s >= a.limit && (int)(x & 0xFFFF) > copies_of(x & 0xFFFF, x >> 16);
  };
  int n_free = 0, n_moves = 0, n_held = 0;
  for (int s = s0; s < s1; s += 64) {
    bool free, moves, held;
    look(s + lane, free, moves, held);
    n_free += __popcll(__ballot(free));
    n_moves += __popcll(__ballot(moves));
    n_held += __popcll(__ballot(held));
  }
  int below = need;                    // wanted by the wave's rows up to this one
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(below, o);
    if (lane >= o) below += u;
  }
  const uint64_t forks = __ballot(fork);
  if (lane == 63) {
    s_sum[w][0] = n_free;
    s_sum[w][1] = n_moves;
    s_sum[w][2] = n_held;
    s_sum[w][3] = below;
    s_sum[w][4] = __popcll(forks);
  }
  __syncthreads();
  int before[5], all[5];
#pragma unroll
  for (int k = 0; k < 5; ++k) {
    before[k] = all[k] = 0;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      if (v < w) before[k] += s_sum[v][k];
      all[k] += s_sum[v][k];
    }
  }
  const int moves_all = all[1];
  const int64_t wanted = (int64_t)moves_all + all[3];
  const int missing = wanted > all[0] ? (int)(wanted - all[0]) : 0;
  if (t == 0) {
    a.info[0] = missing;
    a.info[1] = all[2] + all[3];
    a.info[2] = missing ? 0 : moves_all + all[4];
    a.info[3] = 0;
  }
  if (missing) {
    for (int i = t; i < entries; i += 1024) a.table_out[i] = a.table[i];
    return;
  }
  if (t < a.n_seq) {
    const int at = moves_all + before[3] + below - need;       // number of the row's first wanted slot
    const bool stays = s_edge[t] >= 0 && !fork;
    s_row[t] = mine.end > mine.keep ? make_int4(mine.edge, (mine.end - 1) >> a.cshift, at - mine.edge - stays, stays ? -1 : at)
                                    : make_int4(INT32_MAX, 0, 0, -1);
    s_src[t] = mine.keep & (a.C - 1);
    s_fork[t] = fork ? moves_all + before[4] + rank_of(forks) : -1;
  }
  int f = before[0], mv = before[1];
  for (int s = s0; s < s1; s += 64) {
    bool free, moves, held;
    look(s + lane, free, moves, held);
    const uint64_t fs = __ballot(free), ms = __ballot(moves);
    const int at = f + rank_of(fs), to = mv + rank_of(ms);
    if (free && at < wanted) a.free_at[at] = s + lane;
    if (s + lane < s1) s_slot[s + lane] = moves ? to : -1;
    f += __popcll(fs);
    mv += __popcll(ms);
  }
  __syncthreads();
  for (int s = a.limit + t; s < a.n_slots; s += 1024) {
    const int k = (int)s_slot[s];
    if (k >= 0) a.copies[k] = make_int4(s, a.free_at[k], a.C, 0);
  }
  for (int i0 = t; i0 < entries; i0 += 1024 * PER) {
    int e[PER], at[PER];               // at: the wanted slot's number, -1: none
#pragma unroll
    for (int k = 0; k < PER; ++k) e[k] = a.kept[min(i0 + 1024 * k, entries - 1)];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = min(i0 + 1024 * k, entries - 1), b = row_of(i), c = i - b * a.n_table;
      const int4 row = s_row[b];
      at[k] = e[k] >= a.limit ? (int)s_slot[e[k]] : -1;
      if (c > row.x && c <= row.y) at[k] = row.z + c;
      if (c == row.x && row.w >= 0) {
        at[k] = row.w;
        if (s_fork[b] >= 0 && i0 + 1024 * k < entries) a.copies[s_fork[b]] = make_int4(e[k], a.free_at[at[k]], s_src[b], 0);
      }
    }
    int to[PER];                       // (read by all, so that the loads go out together)
#pragma unroll
    for (int k = 0; k < PER; ++k) to[k] = a.free_at[max(at[k], 0)];
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (i0 + 1024 * k < entries) a.table_out[i0 + 1024 * k] = at[k] >= 0 ? to[k] : e[k];
  }
}

// ---- copies
// A workgroup takes pieces of 256 x 2 times 16 bytes of a (copy, layer): first
// of the key rows, then of the V^T rows, of which a run of 8 positions that
// holds the last one is written value by value.
constexpr int kPiece = 2;

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
        __builtin_nontemporal_store(x[e], reinterpret_cast<f16x8*>(to + off[e]));
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
  if (a.n_slots <= kSmallSlots && a.n_seq <= kSmallRows && entries <= kSmallEntries) {
    hipLaunchKernelGGL(pages_small_kernel, dim3(1), dim3(1024), 0, s, a);
    return;
  }
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
  hipLaunchKernelGGL(kv_copy_kernel, dim3((unsigned)(items < 8192 ? items : 8192)), dim3(256), 0, s, a, pieces);
}

}  // namespace mzk
