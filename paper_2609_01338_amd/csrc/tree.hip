// The trees of drafted tokens of a batch (gfx950): their rows before a step,
// and the branch that is taken after it.
//
// Plan.  A node sees itself and its ancestors.  Each wave takes 64 nodes of a
// tree, a lane each, and follows all parents at once: with M the ancestors of a
// node inside its 64 and n the first of them that is not known yet, M |= M(n), n =
// n(n) doubles what is known, so six steps do.  Then node i's words are M of its
// own 64, M of the first ancestor outside of it, and so on, at most 16 steps
// whatever the depth, and the depth is their bits' number.  It is bound by its launch:
// 2.1 us for one tree of 7 nodes, 3.0 for 64 trees of 61.
//
// Accept.  One wave walks from the root, 64 nodes in a look for the child that holds
// the parent's choice, among the first 1024 nodes, whose parents, tokens and choices
// LDS holds (of a longer chain the next call takes the rest).  Then the keys and
// values move.  Of the keys a thread owns 16 bytes of the rows for all of the branch,
// eight places at a time, read before they are written.  Of V^T a value moves within
// a row of its own, a line of memory for two bytes, so what counts is lines: four
// lanes own the 64 bytes of a dimension that 32 places lie in, and write what
// changes of them as 16 bytes, several layers at a time.  Since path[i] >= i ascends,
// what has been written (places up to i) is never what is still to be read (path[j]
// > i for j > i), so nothing waits for another wave.
//
// The branches of 64 trees of 61 nodes in 32 layers of 8 KV heads of 128 take 69 us.
// A launch that ends behind the walk, which each of 16320 workgroups does for itself,
// takes 15, one behind the slots 17, one that writes no V^T 46: reading 1.2 million lines
// (160 MB) takes 28 and writing as many, of which 2 bytes change (42 MB), 24.  Both
// are 43 at the rate of a large copy.  Whole 64-byte lines are no faster than the 16
// bytes.  So many lines want all channels and many waves: 16384 workgroups (2048: 139), a
// sequence's slices on all XCDs (on one: 87).  One tree of 7 nodes in 16 layers of 8 KV heads of 64 takes 4.3 us.
#include "mz_kernels.h"

namespace mzk {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Rows of sequence b: its first and how many.
__device__ __forceinline__ int tree_rows(const int32_t* row_off, int b, int m, int& first) {
  first = min(max(row_off[b], 0), m);
  return min(max(row_off[b + 1], first), m) - first;
}

__device__ __forceinline__ int tree_len(const int32_t* lens, int b) { return min(max(lens[b], 0), 1 << 30); }

__device__ __forceinline__ void no_tree(const TreePlan& a, int r) {
  if (a.seq) a.seq[r] = -1;
  if (a.place) a.place[r] = -1;
  if (a.rope_pos) a.rope_pos[r] = -1;
  if (a.mask)
    for (int w = 0; w < a.mask_words; ++w) a.mask[(int64_t)r * a.mask_words + w] = 0;
}

__global__ __launch_bounds__(256) void tree_plan_kernel(TreePlan a) {
  __shared__ uint64_t s_seen[kTreeNodes];    // ancestors within a node's 64, itself among them
  __shared__ int s_out[kTreeNodes];          // its first ancestor outside of them, or -1
  const int b = blockIdx.x;
  if (b == a.n_seq) {                        // rows before the first tree and behind the last
    const int before = min(max(a.row_off[0], 0), a.m), last = min(max(a.row_off[a.n_seq], before), a.m);
    for (int i = threadIdx.x; i < before + a.m - last; i += 256) no_tree(a, i < before ? i : last + i - before);
    return;
  }
  int first;
  const int rows = tree_rows(a.row_off, b, a.m, first), len = tree_len(a.lens, b);
  int n = a.mask ? min(rows, 32 * a.mask_words) : rows;
  if (a.parent) n = min(n, kTreeNodes);
  if (a.parent) {
    const int lane = threadIdx.x & 63;
    for (int i0 = threadIdx.x - lane; i0 < n; i0 += 256) {
      const int i = i0 + lane;
      const int p = i < n ? a.parent[first + i] : -1;
      const bool ok = p >= 0 && p < i;
      int next = ok && p >= i0 ? p - i0 : -1, out = ok && p < i0 ? p : -1;
      uint64_t seen = 1ull << lane;
#pragma unroll
      for (int step = 0; step < 6; ++step) {
        const int from = next >= 0 ? next : lane;
        const uint64_t more = __shfl(seen, from);
        const int o = __shfl(out, from), nn = __shfl(next, from);
        if (next >= 0) {
          seen |= more;
          out = o;
          next = nn;
        }
      }
      if (i < n) {
        s_seen[i] = seen;
        s_out[i] = out;
      }
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < rows; i += 256) {
    const int r = first + i;
    if (i >= n) {
      no_tree(a, r);
      continue;
    }
    int depth = i;
    if (a.parent) {
      depth = -1;
      int w = (i >> 6) * 2 + 2;              // words from w on are written
      uint32_t* mask = a.mask + (int64_t)r * a.mask_words;
      if (a.mask)
        for (int v = w; v < a.mask_words; ++v) mask[v] = 0;
      for (int at = i; at >= 0; at = s_out[at]) {
        const uint64_t seen = s_seen[at];
        depth += __popcll(seen);
        if (a.mask) {
          const int own = (at >> 6) * 2;
          for (w -= 2; w > own; w -= 2) {
            mask[w] = 0;
            if (w + 1 < a.mask_words) mask[w + 1] = 0;
          }
          mask[own] = (uint32_t)seen;
          if (own + 1 < a.mask_words) mask[own + 1] = (uint32_t)(seen >> 32);
        }
      }
      if (a.mask)
        for (--w; w >= 0; --w) mask[w] = 0;
    } else if (a.mask) {
      for (int w = 0; w < a.mask_words; ++w)
        a.mask[(int64_t)r * a.mask_words + w] = i >= 32 * w + 31 ? ~0u : i < 32 * w ? 0u : (2u << (i - 32 * w)) - 1;
    }
    if (a.seq) a.seq[r] = b;
    if (a.place) a.place[r] = len + i;
    if (a.rope_pos) a.rope_pos[r] = len + depth;
  }
}

constexpr int kMoves = 8;        // places a thread reads before it writes
constexpr int kLayers = 2;       // layers of V^T likewise

__global__ __launch_bounds__(256) void tree_accept_kernel(TreeAccept a) {
  __shared__ int s_parent[kTreeNodes], s_token[kTreeNodes], s_choice[kTreeNodes], s_path[kTreeNodes];
  // (a sequence's slices follow each other, so that every XCD has some of all sequences)
  const int slices = gridDim.x / a.n_seq, b = blockIdx.x / slices, slice = blockIdx.x - b * slices;
  int first;
  const int rows = tree_rows(a.row_off, b, a.m, first), n = min(rows, kTreeNodes), len = tree_len(a.lens, b);
  const int lane = threadIdx.x & 63;
  int at = n > 0 ? 0 : -1, taken = 0, want = -1, begin = n;      // begin: the first node that moves
  auto take = [&] {
    if (threadIdx.x == 0) s_path[taken] = at;
    if (at != taken) begin = min(begin, taken);
    ++taken;
  };
  if (n <= 64) {
    // every wave walks by itself, a lane a node
    const int i = first + min(lane, max(n - 1, 0));
    int parent = -1, token = -1, choice = -1;
    if (n > 0) {
      parent = a.parent ? a.parent[i] : lane - 1;
      token = a.token[i];
      choice = a.choice[i];
    }
    if (lane >= n || parent >= lane) parent = -1;
    while (at >= 0) {
      take();
      want = __builtin_amdgcn_readlane(choice, at);
      const uint64_t fits = want >= 0 ? __ballot(parent == at && token == want) : 0;
      at = fits ? __builtin_ctzll(fits) : -1;
    }
  } else {
    for (int i = threadIdx.x; i < n; i += 256) {
      const int p = a.parent ? a.parent[first + i] : i - 1;
      s_parent[i] = p < i ? p : -1;
      s_token[i] = a.token[first + i];
      s_choice[i] = a.choice[first + i];
    }
    __syncthreads();
    while (at >= 0) {
      take();
      want = s_choice[at];
      int child = -1;
      if (want >= 0)
        for (int i0 = at & ~63; i0 < n && child < 0; i0 += 64) {
          const int i = i0 + lane;
          const uint64_t fits = __ballot(i < n && s_parent[min(i, n - 1)] == at && s_token[min(i, n - 1)] == want);
          if (fits) child = i0 + __builtin_ctzll(fits);
        }
      at = child;
    }
  }
  if (slice == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    a.accepted[b] = taken;
    a.next[b] = want;
    a.len_out[b] = len + taken;
  }
  __syncthreads();
  if (slice == 0 && blockIdx.y == 0)
    for (int i = threadIdx.x; i < rows; i += 256) a.path[first + i] = i < taken ? s_path[i] : -1;
  if (a.n_layers == 0 || begin >= taken) return;
  // slots that the moves come from in s_parent, -1 where there is none; that they go to in s_token
  const int32_t* table = a.table + (int64_t)b * a.n_table;
  auto slot_at = [&](int pos) {
    const int c = pos >> a.cshift, x = c < a.n_table ? table[c] : -1;
    return (unsigned)x < (unsigned)a.n_slots ? x : -1;
  };
  for (int i = begin + threadIdx.x; i < taken; i += 256) {
    s_token[i] = slot_at(len + i);
    s_parent[i] = s_token[i] >= 0 ? slot_at(len + s_path[i]) : -1;
  }
  __syncthreads();
  const int mask = a.C - 1, v_blocks = (a.dkv + 63) / 64, step = gridDim.y;
  if (slice >= v_blocks) {
    const int item = (slice - v_blocks) * 256 + threadIdx.x, row = a.dkv * 2;
    if (item >= a.dkv / 8) return;
    for (int layer = blockIdx.y; layer < a.n_layers; layer += step) {
      uint8_t* k = a.slab + layer * a.layer_bytes + item * 16;
      for (int i0 = begin; i0 < taken; i0 += kMoves) {
        f16x8 x[kMoves];
#pragma unroll
        for (int e = 0; e < kMoves; ++e) {
          const int i = min(i0 + e, taken - 1), from = s_parent[i];
          if (from >= 0) x[e] = *reinterpret_cast<const f16x8*>(k + from * a.slot_bytes + (int64_t)((len + s_path[i]) & mask) * row);
        }
#pragma unroll
        for (int e = 0; e < kMoves; ++e) {
          const int i = i0 + e;
          if (i < taken && s_parent[i] >= 0)
            *reinterpret_cast<f16x8*>(k + s_token[i] * a.slot_bytes + (int64_t)((len + i) & mask) * row) = x[e];
        }
      }
    }
    return;
  }
  // V^T: lane l of 4 has places pos .. pos + 7 of a dimension, in turns of 32
  const int d = slice * 64 + threadIdx.x / 4;
  if (d >= a.dkv) return;
  const int64_t v_row = (int64_t)(a.dkv + d) * a.C * 2;
  for (int at = (len + begin) & ~31; at < len + taken; at += 32) {
    const int pos = at + (threadIdx.x & 3) * 8;
    const int lo = max(pos, len + begin), hi = min(pos + 8, len + taken);      // places that change
    const int to = lo < hi ? s_token[lo - len] : -1;
    for (int l0 = blockIdx.y; l0 < a.n_layers; l0 += kLayers * step) {
      f16x8 x[kLayers];
#pragma unroll
      for (int y = 0; y < kLayers; ++y) {
        const int layer = l0 + y * step;
        if (to >= 0 && layer < a.n_layers)
          x[y] = *reinterpret_cast<const f16x8*>(a.slab + layer * a.layer_bytes + to * a.slot_bytes + v_row + (pos & mask) * 2);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = pos + e - len;
        if (to < 0 || pos + e < lo || pos + e >= hi || s_parent[i] < 0) continue;
        const int64_t from = s_parent[i] * a.slot_bytes + v_row + ((len + s_path[i]) & mask) * 2;
#pragma unroll
        for (int y = 0; y < kLayers; ++y) {
          const int layer = l0 + y * step;
          if (layer < a.n_layers) x[y][e] = *reinterpret_cast<const _Float16*>(a.slab + layer * a.layer_bytes + from);
        }
      }
      // a lane's values may come from what its neighbours are about to write
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int y = 0; y < kLayers; ++y) {
        const int layer = l0 + y * step;
        if (to >= 0 && layer < a.n_layers)
          *reinterpret_cast<f16x8*>(a.slab + layer * a.layer_bytes + to * a.slot_bytes + v_row + (pos & mask) * 2) = x[y];
      }
    }
  }
}

int accept_slices(int n_layers, int dkv) { return n_layers ? (dkv + 63) / 64 + (dkv / 8 + 255) / 256 : 1; }

}  // namespace

void launch_tree_plan(const TreePlan& a, hipStream_t s) {
  hipLaunchKernelGGL(tree_plan_kernel, dim3(a.n_seq + 1), dim3(256), 0, s, a);
}

bool tree_accept_fits(int n_seq, int n_layers, int dkv) {
  return (int64_t)n_seq * accept_slices(n_layers, dkv) <= kMaxBlocks / 2;
}

void launch_tree_accept(const TreeAccept& a, hipStream_t s) {
  const int64_t blocks = (int64_t)a.n_seq * accept_slices(a.n_layers, a.dkv);
  const int64_t most = blocks < 16384 ? 16384 / blocks : 1;
  const int layers = a.n_layers < 1 ? 1 : a.n_layers < most ? a.n_layers : (int)most;
  hipLaunchKernelGGL(tree_accept_kernel, dim3((unsigned)blocks, layers), dim3(256), 0, s, a);
}

}  // namespace mzk
