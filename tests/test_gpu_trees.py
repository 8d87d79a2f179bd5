"""The calls of a decode step that checks drafted trees -- the rows of the
trees, appending at places apart from rotary positions, the attention of the
trees, the branch that is taken, and the pages of the sequences -- against plain
implementations in 64 bits.

Roundings: U16 = 2^-11 is half a step of f16 relative to the value (2^-25
below its normal range), U32 = 2^-24 half a step of fp32.
"""

import numpy as np
import pytest

from paper_2609_01338_amd import mz
from gpu_util import report, stream, torch_cuda
from test_gpu_batch import TINY16, U16, U32, append_oracle, attention_oracle, attention_run, close, dev, rope_table

pytestmark = pytest.mark.gpu


def ptr(x):
    return 0 if x is None else x.data_ptr()


def offsets(counts, first=0):
    return np.concatenate([[first], first + np.cumsum(counts)]).astype(np.int32)


def random_tree(rng, n, roots=0.0):
    return np.array([-1 if i == 0 or rng.random() < roots else int(rng.integers(max(0, i - 9), i)) for i in range(n)], np.int32)


def full(shape, value=7, dtype=None):
    torch = torch_cuda()
    return torch.full(shape if isinstance(shape, tuple) else (shape,), value, device="cuda", dtype=dtype or torch.int32)


# ----------------------------------------------------------------------------- rows of the trees

def plan_oracle(off, parent, lens, m, words):
    """(seq, place, rope_pos, mask); parent None: chains; words 0: no mask."""
    seq, place, rope = (np.full(m, -1, np.int64) for _ in range(3))
    mask = np.zeros((m, max(words, 1)), np.uint32)
    for b in range(len(lens)):
        n, start = off[b + 1] - off[b], min(max(int(lens[b]), 0), 1 << 30)
        if words:
            n = min(n, 32 * words)
        if parent is not None:
            n = min(n, 1024)
        for i in range(n):
            r, way = off[b] + i, [i]
            while True:
                p = way[-1] - 1 if parent is None else int(parent[off[b] + way[-1]])
                if not 0 <= p < way[-1]:
                    break
                way.append(p)
            seq[r], place[r], rope[r] = b, start + i, start + len(way) - 1
            if words:
                for j in way:
                    mask[r, j // 32] |= np.uint32(1 << j % 32)
    return seq, place, rope, mask


def plan_case(counts, lens, words, seed=0, tree=True, first=0, behind=3, roots=0.1, parent=None):
    rng = np.random.default_rng(seed)
    off = offsets(counts, first)
    m = int(off[-1]) + behind
    if tree and parent is None:
        parent = rng.integers(-5, 5000, m).astype(np.int32)      # rows of no tree hold anything
        for b, n in enumerate(counts):
            parent[off[b]:off[b + 1]] = random_tree(rng, n, roots)
    lens = np.array(lens, np.int32)
    report("plan", counts=list(counts)[:8], words=words, seed=seed, tree=tree)
    d_off, d_lens, d_parent = dev(off), dev(lens), None if parent is None else dev(parent)
    seq, place, rope, mask = full(m), full(m), full(m), full((m, max(words, 1)))
    mz.mz_tree_plan(ptr(d_off), ptr(d_lens), len(lens), m, stream(), parent_ptr=ptr(d_parent), seq_ptr=ptr(seq), place_ptr=ptr(place),
                    rope_pos_ptr=ptr(rope), mask_ptr=ptr(mask) if words else 0, mask_words=words)
    torch_cuda().cuda.synchronize()
    ref = plan_oracle(off, parent, lens, m, words)
    for got, want, what in zip((seq, place, rope), ref, ("seq", "place", "rope_pos")):
        assert np.array_equal(got.cpu().numpy(), want), what
    if words:
        assert np.array_equal(mask.cpu().numpy().view(np.uint32), ref[3]), "mask"


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 128, 200, 257, 1024])
def test_plan_sizes(n):
    plan_case([n, 0, 1, n // 2], [0, 5, 100, 1 << 20], (n + 31) // 32, seed=n)
    plan_case([n, 0, 1, n // 2], [0, 5, 100, 1 << 20], min(32, (n + 31) // 32 + 1), seed=n + 1, first=2, roots=0.5)
    plan_case([n, 3], [7, 9], (n + 31) // 32, tree=False)


def test_plan_deep_and_odd_parents():
    chain = np.arange(-1, 1023).astype(np.int32)
    plan_case([1024], [3], 32, parent=np.concatenate([chain, [4, 4]]).astype(np.int32), behind=2)
    odd = np.array([5, 0, 2, -7, 1, 100, 0], np.int32)      # parents that are the node itself, later ones, none
    plan_case([7], [0], 1, parent=odd, behind=0)


def test_plan_nodes_past_the_mask():
    plan_case([40, 70, 33], [1, 2, 3], 1, seed=3)
    plan_case([40, 70, 33], [1, 2, 3], 2, seed=4, tree=False)
    plan_case([1030, 5], [1, 2], 32, seed=5)
    plan_case([1030, 5], [1, 2], 0, seed=6)


def test_plan_without_mask_and_lengths_out_of_range():
    plan_case([5000, 0, 17], [-3, 2, (1 << 31) - 1], 0, tree=False)
    plan_case([50, 17], [-3, (1 << 30) + 5], 0, seed=7)
    plan_case([0, 0], [1, 1], 1, behind=9)
    plan_case([1] * 700, list(range(700)), 1, seed=8)


def test_plan_single_outputs():
    torch = torch_cuda()
    off, lens, parent = dev(np.array([0, 3], np.int32)), dev(np.array([4], np.int32)), dev(np.array([-1, 0, 0], np.int32))
    for key, want in (("seq_ptr", [0, 0, 0]), ("place_ptr", [4, 5, 6]), ("rope_pos_ptr", [4, 5, 5])):
        got = full(3)
        mz.mz_tree_plan(ptr(off), ptr(lens), 1, 3, stream(), parent_ptr=ptr(parent), **{key: ptr(got)})
        torch.cuda.synchronize()
        assert got.tolist() == want, key


def test_plan_offsets_out_of_range_stay_inside():
    """Offsets that do not ascend within the rows are cut off: what lies outside the buffers is not written."""
    torch = torch_cuda()
    lens = dev(np.array([4, 4, 4], np.int32))
    for off in ([-5, 3, 2, 90], [90, 100, -4, 1 << 30], [0, -(1 << 31), (1 << 31) - 1, 2]):
        seq, room = full(32), dev(np.array(off, np.int32))
        mz.mz_tree_plan(ptr(room), ptr(lens), 3, 8, stream(), seq_ptr=ptr(seq) + 32)
        torch.cuda.synchronize()
        assert (seq[:8] == 7).all() and (seq[16:] == 7).all()


# ----------------------------------------------------------------------------- append by axes

def append_axes_case(nq, nkv, hd, C, f32, axes, pair_axis, seed, m=37, n_rope=200, bad=True):
    torch = torch_cuda()
    rng = np.random.default_rng(seed)
    n_seq, n_table, dkv = 3, 12, nkv * hd
    n_slots = n_seq * n_table + 2
    table = rng.permutation(n_slots)[:n_seq * n_table].reshape(n_seq, n_table).astype(np.int32)
    seq = np.sort(rng.integers(0, n_seq, m)).astype(np.int32)
    pos = np.zeros(m, np.int32)
    for s in range(n_seq):      # places: two runs with a gap
        at = np.nonzero(seq == s)[0]
        pos[at] = int(rng.integers(0, 9)) + np.arange(at.size) + 3 * (np.arange(at.size) > at.size // 2)
    rope_pos = rng.integers(0, n_rope, (axes, m)).astype(np.int32)
    skip = np.zeros(m, bool)
    if bad:
        used = sorted(set(int(x) for x in pair_axis if x != 255))
        seq[1], skip[1] = n_seq, True
        pos[m - 1], skip[m - 1] = n_table * C, True
        if used:
            rope_pos[used[-1], 3], skip[3] = n_rope, True
            rope_pos[used[0], 5], skip[5] = -1, True
    for x in range(axes):      # an axis that no pair turns by may hold anything
        if x not in pair_axis:
            rope_pos[x] = 1 << 30
    rope = rope_table(n_rope, hd)
    dt = np.float32 if f32 else np.float16
    q, k, v = (rng.standard_normal((m, h * hd)).astype(dt) for h in (nq, nkv, nkv))
    slab = rng.standard_normal((n_slots, 2 * C * dkv)).astype(np.float16)
    rows = np.concatenate([q, k, v], 1)
    d = [dev(x) for x in (rows, seq, pos, rope_pos, rope, slab, table)]
    q_out = full((m, nq * hd), 7.0, torch.float16)
    size, wide = rows.itemsize, rows.shape[1]
    base = ptr(d[0])
    report("append_axes", nq=nq, nkv=nkv, hd=hd, C=C, f32=f32, axes=axes, pairs=list(pair_axis)[:12], seed=seed)
    mz.mz_kv_append_axes(m, base + nq * hd * size, base + (nq * hd + dkv) * size, ptr(d[1]), ptr(d[2]), ptr(d[3]), axes, pair_axis,
                         ptr(d[4]), n_rope, ptr(d[5]), n_slots, ptr(d[6]), n_seq, n_table, C, nkv, hd, stream(), q_ptr=base, n_q=nq,
                         q_out_ptr=ptr(q_out), k_stride=wide, v_stride=wide, q_stride=wide, f32=f32)
    torch.cuda.synchronize()
    # the plain append with a rotary row for every row of the batch; a pair that is not turned has (1, 0)
    own = np.zeros((m, hd // 2, 2), np.float32)
    for i, x in enumerate(pair_axis):
        own[:, i] = (1, 0) if x == 255 else rope[np.clip(rope_pos[x], 0, n_rope - 1), i]
    ref, bound = slab.astype(np.float64), np.zeros(slab.shape)
    q_ref, q_bound = np.zeros((m, nq * hd)), np.zeros((m, nq * hd))
    for r in np.nonzero(~skip)[0]:
        # one row, at place 0 of a table of its own chunk
        one = append_oracle(k[r:r + 1], v[r:r + 1], q[r:r + 1] if nq else None, np.zeros(1, int), pos[r:r + 1],
                            np.repeat(own[r:r + 1], pos[r] + 1, 0), slab, table[seq[r]:seq[r] + 1], C, nkv, hd)
        slot, at = table[seq[r], pos[r] // C], pos[r] % C
        where = np.zeros((2, C * dkv), bool)
        where[0].reshape(C, dkv)[at], where[1].reshape(dkv, C)[:, at] = True, True
        where = where.reshape(-1)
        ref[slot, where], bound[slot, where] = one[0][slot, where], one[1][slot, where]
        if nq:
            q_ref[r], q_bound[r] = one[2], one[3]
    close(d[5], ref, bound, "slab")
    if nq:
        close(q_out[dev(~skip)], q_ref[~skip], q_bound[~skip], "q")
        assert bool((q_out[dev(skip)] == 7).all()), "a row that writes nothing"


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 64), (12, 2, 128), (0, 1, 64), (5, 1, 32), (3, 3, 32)])
def test_append_axes_sections(nq, nkv, hd, f32):
    h = hd // 2
    append_axes_case(nq, nkv, hd, 16, f32, 1, [0] * h, seed=hd + nq)
    append_axes_case(nq, nkv, hd, 8, f32, 3, [0] * (h // 4) + [1] * (3 * h // 8) + [2] * (h - h // 4 - 3 * h // 8), seed=hd + nq + 1)
    append_axes_case(nq, nkv, hd, 16, f32, 4, [i % 4 for i in range(h)], seed=hd + nq + 2)
    append_axes_case(nq, nkv, hd, 64, f32, 2, [1] * (h // 2) + [255] * (h - h // 2), seed=hd + nq + 3)
    append_axes_case(nq, nkv, hd, 16, f32, 3, [(0, 2, 255)[i % 3] for i in range(h)], seed=hd + nq + 4)
    append_axes_case(nq, nkv, hd, 16, f32, 1, [255] * h, seed=hd + nq + 5)


@pytest.mark.parametrize("m", [1, 2, 3, 64, 65, 130])
def test_append_axes_rows(m):
    append_axes_case(4, 2, 64, 16, True, 2, [0] * 20 + [1] * 12, seed=m, m=m, bad=m > 6)


def test_append_axes_unturned_pairs_of_infinities():
    """A pair that is not turned holds its two values, whatever the other one is."""
    torch = torch_cuda()
    k = dev(np.array([[np.inf, -np.inf] + [1.5] * 30 + [3.0, np.nan] + [2.5] * 30], np.float32))
    v, zero, slab = torch.zeros(1, 64, device="cuda"), dev(np.zeros((1, 1), np.int32)), torch.zeros(1, 2 * 8 * 64, device="cuda", dtype=torch.float16)
    rope = dev(rope_table(1, 64))
    mz.mz_kv_append_axes(1, ptr(k), ptr(v), ptr(zero), ptr(zero), ptr(zero), 1, [255] * 32, ptr(rope), 1, ptr(slab), 1, ptr(zero), 1, 1, 8,
                         1, 64, stream())
    torch.cuda.synchronize()
    assert np.array_equal(slab[0, :64].float().cpu().numpy(), k[0].cpu().numpy(), equal_nan=True)


@pytest.mark.parametrize("f32", [True, False])
def test_append_axes_has_the_bits_of_append(f32):
    torch = torch_cuda()
    rng = np.random.default_rng(5)
    nq, nkv, hd, C, m, n_rope = 12, 2, 128, 16, 77, 400
    dt = np.float32 if f32 else np.float16
    q, k, v = (dev(rng.standard_normal((m, h * hd)).astype(dt)) for h in (nq, nkv, nkv))
    seq, pos = dev(np.zeros(m, np.int32)), dev((100 + np.arange(m)).astype(np.int32))
    rope, table = dev(rope_table(n_rope, hd)), dev(rng.permutation(32).astype(np.int32)[None])
    out = []
    for axes in (False, True):
        slab, q_out = torch.zeros(32, 2 * C * nkv * hd, device="cuda", dtype=torch.float16), torch.zeros(m, nq * hd, device="cuda", dtype=torch.float16)
        kw = dict(q_ptr=ptr(q), n_q=nq, q_out_ptr=ptr(q_out), f32=f32)
        rest = (ptr(rope), n_rope, ptr(slab), 32, ptr(table), 1, 32, C, nkv, hd, stream())
        if axes:
            mz.mz_kv_append_axes(m, ptr(k), ptr(v), ptr(seq), ptr(pos), ptr(pos), 1, [0] * (hd // 2), *rest, **kw)
        else:
            mz.mz_kv_append(m, ptr(k), ptr(v), ptr(seq), ptr(pos), *rest, **kw)
        torch.cuda.synchronize()
        out.append((slab, q_out))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


# ----------------------------------------------------------------------------- attention of the trees

def tree_inputs(counts, lens, C, nq, nkv, hd, seed, first=0, behind=2, spread=1.0, words=None, mask="tree", extra_table=2):
    """Slots hold NaN past the last key; mask: "tree", "any" (any set of nodes, none among them) or None."""
    rng = np.random.default_rng(seed)
    off, lens = offsets(counts, first), np.array(lens, np.int32)
    m, group, dkv = int(off[-1]) + behind, nq // nkv, nkv * hd
    keys = [max(int(n), 0) + int(t) for n, t in zip(lens, counts)]
    n_table = max(max(keys), 1) // C + 1 + extra_table
    n_slots = sum((n + C - 1) // C for n in keys) + 2
    order, at = rng.permutation(n_slots), 0
    table = rng.integers(-(1 << 31), 1 << 31, (len(lens), n_table)).astype(np.int32)   # entries past a length are never followed
    slab = np.full((n_slots, 2, C * dkv), np.nan, np.float16)                          # nor what slots hold past it
    for b, n in enumerate(keys):
        c = (n + C - 1) // C
        table[b, :c] = order[at:at + c]
        at += c
        for i, slot in enumerate(table[b, :c]):
            t = min(C, n - i * C)
            slab[slot, 0].reshape(C, dkv)[:t] = rng.standard_normal((t, dkv)) * spread
            slab[slot, 1].reshape(dkv, C)[:, :t] = rng.standard_normal((dkv, t))
    q = (rng.standard_normal((m, nq * hd)) * spread).astype(np.float16)
    q[:first], q[off[-1]:] = np.nan, np.nan
    bits = None
    if mask:
        words = words or (max(max(counts), 1) + 31) // 32
        bits = rng.integers(0, 1 << 32, (m, words), dtype=np.uint64).astype(np.uint32)
        if mask == "tree":
            parent = np.full(m, -1, np.int32)
            for b, n in enumerate(counts):
                parent[off[b]:off[b + 1]] = random_tree(rng, n, 0.05)
            bits = plan_oracle(off, parent, lens, m, words)[3]
        else:
            bits[rng.random(m) < 0.3] = 0
    return dict(q=q, off=off, lens=lens, slab=slab.reshape(n_slots, -1), table=table, mask=bits, C=C, nq=nq, nkv=nkv, hd=hd)


def tree_oracle(a, lens=None, off=None):
    """(out, bound, rows that are written)."""
    q, slab, table, mask, C, nq, nkv, hd = (a[k] for k in ("q", "slab", "table", "mask", "C", "nq", "nkv", "hd"))
    off, lens = a["off"] if off is None else off, a["lens"] if lens is None else lens
    m, n_slots, dkv, group = q.shape[0], slab.shape[0], nkv * hd, nq // nkv
    out, bound, wrote = np.zeros((m, nq * hd)), np.zeros((m, nq * hd)), np.zeros(m, bool)
    halves = slab.reshape(n_slots, 2, C * dkv)
    ks, vs = halves[:, 0].reshape(n_slots, C, dkv), halves[:, 1].reshape(n_slots, dkv, C)
    top = table.shape[1] * C
    for b in range(len(lens)):
        t = int(off[b + 1] - off[b])
        if mask is not None:
            t = min(t, 32 * mask.shape[1])
        n = min(max(int(lens[b]), 0), top)
        end = min(n + t, top)
        at = np.array([j for j in range(end) if 0 <= int(table[b, j // C]) < n_slots], int)
        wrote[off[b]:off[b] + t] = True
        if at.size == 0:
            continue
        slots = table[b, at // C]
        k, v = ks[slots, at % C].astype(np.float64).reshape(-1, nkv, hd), vs[slots, :, at % C].astype(np.float64).reshape(-1, nkv, hd)
        for i in range(t):
            r = off[b] + i
            see = at < n
            node = np.clip(at - n, 0, None)
            see |= (at >= n) & ((node <= i) if mask is None else ((mask[r, node // 32] >> (node % 32).astype(np.uint32)) & 1).astype(bool))
            if not see.any():
                continue
            for h in range(nq):
                x = q[r, h * hd:(h + 1) * hd].astype(np.float64)
                kk, vv = k[see, h // group], v[see, h // group]
                with np.errstate(invalid="ignore", over="ignore"):
                    s = kk @ x / np.sqrt(hd)
                    w = np.exp(s - s.max())
                    p = w / w.sum()
                    o = p @ vv
                    on = np.isfinite(s)
                    if on.any():
                        # the score's sum of hd exact products and its scale, the exponent, exp2 (1 ulp): e on each weight,
                        # once above and once below the line; 22 bits of a weight; sums of n terms in runs of 32 and the
                        # factors of the running max; the lower half of a weight is within 2^-25 of 2^11 times the largest at the least,
                        # below its normal range: 2^-36
                        part = (np.abs(kk[on]) @ np.abs(x)).max() / np.sqrt(hd)
                        e = (hd + 4) * U32 * part + 4 * U32 * np.abs(s[on] - s[on].max()).max() + 4 * U32
                        size = p[on] @ np.abs(vv[on])
                        bound[r, h * hd:(h + 1) * hd] = (2 * e + 2.0 ** -21 + 8 * (len(s) / 32 + 64) * U32) * size * (1 + U16) + \
                            U16 * np.abs(o) + TINY16 + len(s) * 2.0 ** -36 * np.abs(vv[on]).max(0)
                out[r, h * hd:(h + 1) * hd] = o
    return out, bound, wrote


def tree_run(a, d=None, ws=None, out=None, lens=None, off=None):
    torch = torch_cuda()
    d = d or {k: (None if a[k] is None else dev(a[k])) for k in ("q", "off", "lens", "slab", "table", "mask")}
    m, n_seq = a["q"].shape[0], len(a["lens"])
    need = mz.mz_attention_tree_workspace_bytes(m, n_seq, a["nq"], a["nkv"], a["hd"])
    if ws is None:
        ws = torch.full((need // 4 + 1,), float("nan"), device="cuda")      # what it held must not show
    if out is None:
        out = full((m, a["nq"] * a["hd"]), 7.0, torch.float16)
    mask = {} if a["mask"] is None else dict(mask_ptr=ptr(d["mask"]), mask_words=a["mask"].shape[1])
    mz.mz_attention_tree(ptr(d["q"]), m, ptr(d["off"]), ptr(d["lens"]), n_seq, ptr(d["slab"]), d["slab"].shape[0], ptr(d["table"]),
                         d["table"].shape[1], a["C"], a["nq"], a["nkv"], a["hd"], ptr(ws), need, ptr(out), stream(), **mask)
    return out


def tree_check(a, out, what="out", **kw):
    torch_cuda().cuda.synchronize()
    ref, bound, wrote = tree_oracle(a, **kw)
    close(out[dev(wrote)], ref[wrote], bound[wrote], what)
    assert bool((out[dev(~wrote)] == 7).all()), what + ": rows of no tree"


def tree_case(*args, **kw):
    a = tree_inputs(*args, **kw)
    report("attention_tree", counts=list(args[0])[:8], lens=list(args[1])[:8], C=a["C"], nq=a["nq"], nkv=a["nkv"], hd=a["hd"],
           mask=None if a["mask"] is None else a["mask"].shape, seed=kw.get("seed"))
    out = tree_run(a)
    tree_check(a, out)
    assert torch_cuda().equal(tree_run(a), out), "another run, other bits"
    return a, out


HEADS = [(4, 2, 64), (8, 8, 128), (12, 2, 128), (16, 1, 64), (32, 8, 64), (5, 1, 128)]


@pytest.mark.parametrize("mask", ["tree", "any", None])
@pytest.mark.parametrize("nq,nkv,hd", HEADS)
def test_tree_attention_heads(nq, nkv, hd, mask):
    for C in (8, 16, 64):
        tree_case([1, 6, 0, 3], [40, 0, 17, 129], C, nq, nkv, hd, seed=C + nq, mask=mask)


@pytest.mark.parametrize("mask", ["tree", None])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100])
def test_tree_attention_nodes(n, mask):
    tree_case([n], [77], 16, 4, 2, 64, seed=n, mask=mask)
    tree_case([n, 1, n], [0, 300, 31], 64, 6, 1, 128, seed=n + 1, mask=mask, first=1)


@pytest.mark.parametrize("n", [0, 1, 7, 8, 31, 32, 33, 95, 96, 120, 121, 127, 128, 129, 255, 256, 700])
def test_tree_attention_lengths(n):
    """Trees that begin anywhere in a lane's eight keys, a block and a unit."""
    tree_case([9, 5], [n, n + 3], 8, 4, 2, 64, seed=n, mask="any")
    tree_case([35, 5], [n, n + 3], 32, 2, 1, 128, seed=n + 1, mask="any")


@pytest.mark.parametrize("nq,hd", [(2, 64), (16, 128)])
def test_tree_attention_offsets_that_descend(nq, hd):
    """Rows of several sequences at once, whose units would pass 31 bits: no row is written.  (No chunk has a slot,
    so that nothing is to be read in any case.)"""
    torch = torch_cuda()
    m, C = 1024, 256
    for n_seq, n_table, off in ((3, 4, [0, 5, 3, 8]), (3, 4, [0, 8, 8, 7]), (700, 4, [0] * 256 + [9, 8] + [9] * 443),
                                (2048, 16384 // (nq // 2), [0, m] * 1024 + [0]), (300, 32768, [0, m] * 150 + [0])):
        report("attention_tree", n_seq=n_seq, n_table=n_table, off=off[:8], nq=nq, hd=hd)
        assert len(off) == n_seq + 1
        table = full((n_seq, n_table), -1)
        lens = full(n_seq, n_table * C - 100)
        q, slab = full((m, nq * hd), 1.0, torch.float16), full((1, 2 * C * hd), 1.0, torch.float16)
        need = mz.mz_attention_tree_workspace_bytes(m, n_seq, nq, 1, hd)
        ws, out, d_off = torch.full((need // 4 + 1,), float("nan"), device="cuda"), full((m, nq * hd), 7.0, torch.float16), dev(np.array(off, np.int32))
        mz.mz_attention_tree(ptr(q), m, ptr(d_off), ptr(lens), n_seq, ptr(slab), 1, ptr(table), n_table, C, nq, 1, hd, ptr(ws), need, ptr(out), stream())
        torch.cuda.synchronize()
        assert bool((out == 7).all())
    d_off.copy_(dev(np.minimum(np.arange(n_seq + 1), m).astype(np.int32)))      # the same workspace, offsets that ascend: no key has a slot
    mz.mz_attention_tree(ptr(q), m, ptr(d_off), ptr(lens), n_seq, ptr(slab), 1, ptr(table), n_table, C, nq, 1, hd, ptr(ws), need, ptr(out), stream())
    torch.cuda.synchronize()
    assert not bool(out[:n_seq].any()) and bool((out[n_seq:] == 7).all())      # (the rows behind are of no tree)


@pytest.mark.parametrize("C", [8, 32, 256])
def test_tree_attention_shared_by_many_workgroups(C):
    tree_case([3, 1, 5], [9000, 40, 6100], C, 4, 2, 64, seed=C)
    tree_case([20, 1], [5000, 3000], C, 4, 1, 128, seed=C + 1)


def test_tree_attention_of_1024_nodes():
    tree_case([1024], [50], 64, 2, 2, 64, seed=1, mask="any", behind=0)
    tree_case([1100, 3], [10, 20], 64, 1, 1, 64, seed=2, mask="any", words=32)      # nodes past the mask are rows of no tree


def test_tree_attention_nodes_past_the_mask():
    tree_case([40, 70, 2], [12, 0, 33], 16, 4, 2, 64, seed=3, mask="any", words=1)
    tree_case([40, 70, 2], [12, 0, 33], 16, 4, 2, 64, seed=3, mask="any", words=5)


def test_tree_attention_long_chain():
    tree_case([1500, 4], [100, 0], 64, 2, 1, 64, seed=4, mask=None)


def test_tree_attention_no_sequence_has_rows():
    tree_case([0, 0], [5, 9], 16, 4, 2, 64, seed=5, behind=4)


def test_tree_attention_no_sequence_has_rows_after_other_work():
    """Nor is anything of what a workgroup's LDS held before taken for a sequence: wide and few columns."""
    for nq, nkv, hd, behind in ((4, 2, 64, 4), (16, 1, 128, 40), (32, 2, 64, 700)):
        tree_case([3, 60, 1], [500, 90, 7], 16, nq, nkv, hd, seed=nq)
        tree_case([0, 0, 0], [5, 9, 0], 16, nq, nkv, hd, seed=5, behind=behind)


def test_tree_attention_padded_batch():
    """Few of many sequences have rows."""
    counts, lens = np.zeros(700, int), np.zeros(700, int)
    for b, t, n in ((0, 2, 100), (3, 5, 0), (300, 1, 1000), (699, 4, 50)):
        counts[b], lens[b] = t, n
    tree_case(counts, lens, 16, 4, 2, 64, seed=6, mask="any")


def test_tree_attention_many_sequences_of_wide_trees():
    """More sequences than a workgroup has threads, most of them with as many rows as make wide tiles."""
    rng = np.random.default_rng(7)
    counts, lens = rng.integers(17, 40, 300), rng.integers(0, 90, 300)
    counts[rng.integers(0, 300, 40)] = 0
    tree_case(counts, lens, 16, 4, 2, 64, seed=60, mask="tree")
    tree_case(counts, lens, 64, 4, 2, 64, seed=61, mask=None)


@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 64), (2, 2, 64), (8, 1, 128)])
@pytest.mark.parametrize("rest", [1, 0])
def test_tree_attention_a_piece_beside_many_short_sequences(rest, nq, nkv, hd):
    """Tiles go by the average of the rows, far from any sequence's own."""
    rng = np.random.default_rng(nq + rest)
    counts, lens = np.full(40, rest), rng.integers(0, 500, 40)
    counts[[7, 39]], lens[[7, 39]] = (130, 40), (900, 0)
    tree_case(counts, lens, 16, nq, nkv, hd, seed=80, mask=None)
    tree_case(counts, lens, 64, nq, nkv, hd, seed=81, mask="tree")


def test_tree_attention_a_row_that_sees_nothing():
    a = tree_inputs([4, 3], [0, 0], 16, 4, 2, 64, seed=7, mask="any")
    a["mask"][:] = 0
    a["mask"][2] = 4
    out = tree_run(a)
    tree_check(a, out)
    assert not out[[0, 1, 3]].any() and out[2].any()


def test_tree_attention_lengths_out_of_range():
    a = tree_inputs([4, 3, 2], [20, 0, 60], 16, 4, 2, 64, seed=8, mask="any", extra_table=0)
    top = a["table"].shape[1] * 16
    for b in (0, 2):      # tables of full chunks
        a["table"][b] = np.arange(a["table"].shape[1])
    a["slab"] = np.nan_to_num(a["slab"])
    for lens in ([-5, 0, 60], [top, 0, top - 1], [(1 << 31) - 1, -(1 << 31), top + 1]):
        a["lens"] = np.array(lens, np.int32)
        tree_check(a, tree_run(a), f"lengths {lens}")


def test_tree_attention_chunks_without_a_slot():
    for C in (8, 32, 64):
        a = tree_inputs([20, 6, 3], [300, 100, 2], C, 4, 2, 64, seed=9, mask="any")
        a["table"][0, [0, 2, 300 // C]] = (-1, 1 << 30, a["slab"].shape[0])
        a["table"][2, 0] = -7      # all of a sequence's keys
        tree_check(a, tree_run(a), f"chunks of {C}")


@pytest.mark.parametrize("nq,nkv", [(4, 2), (16, 1)])
def test_tree_attention_of_many_sequences_with_infinite_values(nq, nkv):
    """Rows cut over several shares, far behind in a batch of which few sequences have rows, are taken again."""
    counts, lens = np.zeros(150000, int), np.zeros(150000, int)
    for b, t, n in ((0, 2, 100), (3, 5, 6000), (70001, 1, 9000), (149998, 4, 8000), (149999, 1, 70)):
        counts[b], lens[b] = t, n
    a = tree_inputs(counts, lens, 256, nq, nkv, 64, seed=64, mask="tree")
    for b, at, d in ((3, 17, 2), (70001, 8999, 5), (149998, 4000, 60), (149998, 8001, 9)):
        a["slab"][a["table"][b, at // 256]].reshape(2, -1)[1].reshape(-1, 256)[d, at % 256] = np.inf
    report("attention_tree", n_seq=len(lens), nq=nq, nkv=nkv)
    out = tree_run(a)
    tree_check(a, out)
    assert np.isinf(out.cpu().numpy()[:13]).sum() >= 5 * nq // nkv


@pytest.mark.parametrize("C", [8, 64])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_tree_attention_what_a_row_does_not_see(bad, C):
    """NaN and infinities in nodes that only some rows see: in the output of those, and of no other."""
    a = tree_inputs([12, 5], [40, 7], C, 4, 2, 64, seed=10, mask="tree")
    dkv = 128
    for b, node, half in ((0, 3, 1), (0, 7, 0), (1, 2, 1), (1, 4, 0)):
        at = a["lens"][b] + node
        slot = a["table"][b, at // C]
        if half:
            a["slab"][slot].reshape(2, -1)[1].reshape(dkv, C)[5:70, at % C] = bad
        else:
            a["slab"][slot].reshape(2, -1)[0].reshape(C, dkv)[at % C, 3] = bad
    with np.errstate(invalid="ignore"):
        ref, _, _ = tree_oracle(a)
    hit = ~np.isfinite(ref).all(1)
    assert hit.any() and not hit[:17].all()
    tree_check(a, tree_run(a), f"{bad}")


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("C,n", [(8, 30), (64, 200), (64, 5000), (16, 4000)])
def test_tree_attention_wide_trees_and_what_a_row_does_not_see(C, n, bad):
    """The same for trees of many columns, alone in a workgroup's share and cut over several."""
    a = tree_inputs([24, 9], [n, 7], C, 8, 1, 64, seed=C + n, mask="tree")
    for b, node, half in ((0, 5, 1), (0, 17, 0), (1, 2, 1)):
        at = a["lens"][b] + node
        slot = a["table"][b, at // C]
        if half:
            a["slab"][slot].reshape(2, -1)[1].reshape(64, C)[3:40, at % C] = bad
        else:
            a["slab"][slot].reshape(2, -1)[0].reshape(C, 64)[at % C, 3] = bad
    with np.errstate(invalid="ignore"):
        ref, _, _ = tree_oracle(a)
    hit = ~np.isfinite(ref[:33]).all(1)
    assert hit.any() and not hit.all()
    tree_check(a, tree_run(a), f"{bad}")


@pytest.mark.parametrize("counts,lens,nq,nkv,hd,C", [
    ([12, 5], [40, 7], 4, 2, 64, 16), ([12, 5], [40, 7], 12, 2, 128, 64), ([6, 5], [9000, 40], 4, 2, 64, 64), ([9, 3], [5000, 40], 6, 2, 128, 8),
    ([24, 9], [30, 7], 8, 1, 64, 8), ([40, 20], [200, 7], 4, 2, 64, 64), ([40, 30], [5000, 7], 4, 2, 64, 64), ([21, 9], [4000, 7], 6, 1, 128, 16)])
def test_tree_attention_bits_of_rows_that_do_not_see_a_key_of_nan(counts, lens, nq, nkv, hd, C):
    """A key of NaN changes the rows that see it, in its head, and not a bit of the others: few and many columns, alone in
    a workgroup's share and cut over several."""
    a = tree_inputs(counts, lens, C, nq, nkv, hd, seed=C + nq, mask="tree")
    clean = tree_run(a).cpu().numpy()
    sees = np.zeros((len(a["q"]), nq), bool)
    for b, node in ((0, 3), (1, 2)):
        at = a["lens"][b] + node
        a["slab"][a["table"][b, at // C]].reshape(2, -1)[0].reshape(C, nkv * hd)[at % C, 3] = np.nan
        sees[a["off"][b]:a["off"][b + 1], :nq // nkv] = ((a["mask"][a["off"][b]:a["off"][b + 1], 0] >> node) & 1)[:, None].astype(bool)
    got = tree_run(a)
    tree_check(a, got)
    got, sees = got.cpu().numpy(), np.repeat(sees, hd, 1)
    assert sees.any() and not sees[:a["off"][-1], :(nq // nkv) * hd].all()
    assert np.isnan(got[sees]).all()
    assert np.array_equal(got[~sees].view(np.uint16), clean[~sees].view(np.uint16))


@pytest.mark.parametrize("C", [8, 64, 256])
def test_tree_attention_a_value_that_all_rows_see_is_infinite(C):
    a = tree_inputs([24, 9], [700, 7], C, 8, 1, 64, seed=C, mask="any")
    slot = a["table"][0, 300 // C]
    a["slab"][slot].reshape(2, -1)[1].reshape(64, C)[11, 300 % C] = np.inf
    tree_check(a, tree_run(a))


@pytest.mark.parametrize("C", [8, 64, 512])
def test_tree_attention_of_two_million_keys(C):
    """Shares of more tiles than their copy of the chunk table holds at once."""
    torch = torch_cuda()
    n, t, nq, hd = 2200000, 3, 16, 64
    chunks = (n + t + C - 1) // C
    g = torch.Generator(device="cuda").manual_seed(C)
    table = torch.randperm(chunks, device="cuda", generator=g).int()[None]
    slab = torch.empty(chunks, 2, C * hd, device="cuda", dtype=torch.float16).normal_(generator=g)
    q = torch.empty(t, nq * hd, device="cuda", dtype=torch.float16).normal_(generator=g)
    off, lens = dev(np.array([0, t], np.int32)), dev(np.array([n], np.int32))
    ws = torch.empty(mz.mz_attention_tree_workspace_bytes(t, 1, nq, 1, hd), device="cuda", dtype=torch.uint8)
    out = full((t, nq * hd), 7.0, torch.float16)
    mz.mz_attention_tree(ptr(q), t, ptr(off), ptr(lens), 1, ptr(slab), chunks, ptr(table), chunks, C, nq, 1, hd, ptr(ws), ws.numel(), ptr(out),
                         stream())
    at = table[0].long()
    k = slab[at, 0].view(-1, hd)[:n + t].double()
    v = slab[at, 1].view(-1, hd, C).transpose(1, 2).reshape(-1, hd)[:n + t].double()
    s = q.view(-1, hd).double() @ k.T.contiguous() / 8
    s.masked_fill_(torch.arange(n + t, device="cuda")[None, :] > n + torch.arange(t * nq, device="cuda")[:, None] // nq, -np.inf)
    p = torch.softmax(s, 1)
    ref = (p @ v).cpu().numpy().reshape(t, nq * hd)
    # as tree_oracle's; a score is at most |q| |k| / 8, a share's sums have at most 8192 terms of a column, and 512 are joined
    size = (p @ v.abs()).cpu().numpy().reshape(t, nq * hd)
    part = float((q.view(-1, hd).double().norm(dim=1).max() * k.norm(dim=1).max()) / 8)
    e = (hd + 4) * U32 * part + 4 * U32 * 2 * part + 4 * U32
    bound = (2 * e + 2.0 ** -21 + 8 * (8192 / 32 + 512 + 64) * U32) * size * (1 + U16) + U16 * np.abs(ref) + TINY16 + n * 2.0 ** -34 * float(v.abs().max()) * \
        float(p.max())
    close(out, ref, bound, "out")


def test_tree_attention_large_scores():
    tree_case([8, 3], [200, 31], 16, 4, 2, 64, seed=11, spread=30.0)


def test_tree_attention_cancelling_values():
    """Values that are all but each other's opposite: a weight's rounding to f16 would show."""
    a = tree_inputs([6], [500], 16, 4, 2, 64, seed=12, spread=0.02)
    halves = a["slab"].reshape(a["slab"].shape[0], 2, 128, 16)
    halves[:, 1] = np.where(np.isnan(halves[:, 1]), np.nan, np.where(np.arange(16) % 2 == 0, 1.0, -1.0))
    tree_check(a, tree_run(a))


def test_tree_attention_of_one_node_is_the_batched_step():
    a = tree_inputs([1, 1, 1], [50, 700, 0], 16, 8, 2, 128, seed=13, mask=None, behind=0)
    out = tree_run(a)
    one = attention_run(a["q"], a["lens"] + 1, a["slab"], a["table"], 16, 8, 2, 128)
    ref, bound = attention_oracle(a["q"], a["lens"] + 1, a["slab"], a["table"], 16, 8, 2, 128)
    close(out, ref, bound, "tree")
    close(one, ref, bound, "batch")


def test_tree_attention_far_slots():
    """Slots past 2^32 bytes of the slab."""
    torch = torch_cuda()
    C, nq, nkv, hd = 64, 4, 2, 128
    a = tree_inputs([5, 2], [150, 64], C, nq, nkv, hd, seed=14, mask="any")
    n_slots = (1 << 32) // (C * nkv * hd * 4) + 40
    slab = torch.full((n_slots, 2 * C * nkv * hd), float("nan"), device="cuda", dtype=torch.float16)
    far = n_slots - a["slab"].shape[0]
    slab[far:] = dev(a["slab"])
    table = a["table"].copy()
    for b in range(2):
        c = (int(a["lens"][b]) + (5, 2)[b] + C - 1) // C
        table[b, :c] += far
    d = dict(q=dev(a["q"]), off=dev(a["off"]), lens=dev(a["lens"]), slab=slab, table=dev(table), mask=dev(a["mask"]))
    tree_check(a, tree_run(a, d))


# The same for trees of so many columns that tiles of 128 are taken: (nq, nkv, hd).
WIDE_HEADS = [(8, 1, 64), (12, 2, 128), (32, 2, 64)]


def wide_inputs(counts, lens, C, heads, **kw):
    """tree_inputs whose average sequence has more than 32 columns: rows and heads of a KV head."""
    a = tree_inputs(counts, lens, C, *heads, **kw)
    assert -(-len(a["q"]) // len(counts)) * (heads[0] // heads[1]) > 32
    return a


@pytest.mark.parametrize("heads", WIDE_HEADS)
@pytest.mark.parametrize("C", [8, 32, 64, 256])
def test_wide_trees_chunks_without_a_slot(C, heads):
    """Missing first, middle, last and neighbouring chunks, the trees' own, and all of a sequence; one share and many."""
    for n, seed in ((300, 70), (700, 71), (6000, 72)):
        a = wide_inputs([24, 9, 5], [n, 100, 2], C, heads, seed=seed + C, mask="any")
        a["table"][0, [0, n // 2 // C, n // 2 // C + 1, n // C]] = (-1, 1 << 30, a["slab"].shape[0], -(1 << 31))
        a["table"][1, 70 // C] = -3
        a["table"][2] = -7
        out = tree_run(a)
        tree_check(a, out, f"chunks of {C}, {n} keys")
        assert not out[33:38].any()


@pytest.mark.parametrize("heads", WIDE_HEADS)
@pytest.mark.parametrize("C", [16, 64])
def test_wide_trees_lengths_out_of_range(C, heads):
    a = wide_inputs([24, 13, 2], [220, 0, 460], C, heads, seed=73, mask="any", extra_table=0)
    wide = a["table"].shape[1]
    for b in (0, 2):      # tables of full chunks
        a["table"][b] = np.arange(wide) % a["slab"].shape[0]
    a["table"][1] = np.where((a["table"][1] >= 0) & (a["table"][1] < a["slab"].shape[0]), a["table"][1], 0)
    a["slab"], top = np.nan_to_num(a["slab"]), wide * C
    for lens in ([-5, 0, 60], [top, 0, top - 1], [(1 << 31) - 1, -(1 << 31), top + 1], [top - 9, top - 64, top - 65]):
        a["lens"] = np.array(lens, np.int32)
        tree_check(a, tree_run(a), f"lengths {lens}")


@pytest.mark.parametrize("C", [16, 64])
@pytest.mark.parametrize("heads", [(8, 1, 128), (32, 2, 64)])
def test_wide_trees_far_slots(C, heads):
    """Slots past 2^32 bytes of the slab."""
    torch = torch_cuda()
    a = wide_inputs([25, 9], [1500, 64], C, heads, seed=74, mask="any")
    n_slots = (1 << 32) // (C * heads[1] * heads[2] * 4) + a["slab"].shape[0] + 9
    slab = torch.full((n_slots, 2 * C * heads[1] * heads[2]), float("nan"), device="cuda", dtype=torch.float16)
    far = n_slots - a["slab"].shape[0]
    slab[far:] = dev(a["slab"])
    table = a["table"].copy()
    for b in range(2):
        c = (int(a["lens"][b]) + (25, 9)[b] + C - 1) // C
        table[b, :c] += far
    tree_check(a, tree_run(a, dict(q=dev(a["q"]), off=dev(a["off"]), lens=dev(a["lens"]), slab=slab, table=dev(table), mask=dev(a["mask"]))))


@pytest.mark.parametrize("heads", WIDE_HEADS)
@pytest.mark.parametrize("C", [16, 128])
def test_wide_trees_large_scores(C, heads):
    a = wide_inputs([24, 13], [500, 31], C, heads, seed=75, spread=30.0)
    tree_check(a, tree_run(a))


@pytest.mark.parametrize("counts,lens,heads", [([7, 2], [900, 30], (4, 2, 64)), ([24, 13], [900, 30], (8, 1, 64)), ([24, 13], [900, 5000], (12, 2, 128))])
@pytest.mark.parametrize("way", ["up", "down", "steps", "one at the end"])
def test_tree_attention_scores_that_rise_along_the_keys(counts, lens, heads, way):
    """The largest score grows by less and by more than what a running maximum may fall behind, or comes last."""
    C = 32
    a = tree_inputs(counts, lens, C, *heads, seed=76, mask=None)
    nq, nkv, hd = heads
    a["q"][:] = np.random.default_rng(77).uniform(0.5, 1.0, a["q"].shape)
    dkv = nkv * hd
    for b, n in enumerate(np.array(lens) + counts):
        j = np.arange(n)
        high = {"up": j / n, "down": 1 - j / n, "steps": (j // 70) % 5 / 5 + (j // 350) / 20, "one at the end": (j == n - 1) * 1.0}[way] * 12 / np.sqrt(hd)
        for i, slot in enumerate(a["table"][b, :(n + C - 1) // C]):
            t = min(C, n - i * C)
            a["slab"][slot].reshape(2, -1)[0].reshape(C, dkv)[:t] = high[i * C:i * C + t, None]
    tree_check(a, tree_run(a))


@pytest.mark.parametrize("counts,lens,heads", [([6, 3], [400, 31], (4, 2, 64)), ([3, 2], [700, 31], (4, 1, 128)),
                                               ([24, 13], [300, 31], (8, 1, 64)), ([24, 13], [900, 31], (8, 1, 128)), ([33], [2000], (8, 1, 128))])
@pytest.mark.parametrize("C", [16, 64, 256])
def test_tree_attention_lower_halves_of_the_weights(C, counts, lens, heads):
    """Two kinds of keys in turn, with values of 1 and -1: a weight's rounding to f16 is the same for all keys of a kind and stays
    in the sum.  The same sums with weights of f16 lie outside of the bound, which so holds the further bits."""
    a = tree_inputs(counts, lens, C, *heads, seed=78, mask=None, behind=0)
    (nq, nkv, hd), rng = heads, np.random.default_rng(79)
    kinds = (rng.standard_normal((2, nkv * hd)) * 0.05).astype(np.float16)
    for b, n in enumerate(np.array(lens) + counts):
        for i, slot in enumerate(a["table"][b, :(n + C - 1) // C]):
            t = min(C, n - i * C)
            k, v = a["slab"][slot].reshape(2, -1)
            k.reshape(C, -1)[:t] = kinds[np.arange(t) % 2]
            v.reshape(-1, C)[:, :t] = np.where(np.arange(t) % 2 == 0, 1.0, -1.0)
    ref, bound, _ = tree_oracle(a)
    tree_check(a, tree_run(a))
    worst = 0.0
    for b, n in enumerate(lens):
        for i in range(counts[b]):
            r = a["off"][b] + i
            for h in range(nq):
                x, g = a["q"][r, h * hd:(h + 1) * hd].astype(np.float64), h // (nq // nkv) * hd
                s = kinds[:, g:g + hd].astype(np.float64) @ x / np.sqrt(hd)
                w, times = 2.0 ** 11 * np.exp(s - s.max()), np.array([(n + i + 2) // 2, (n + i + 1) // 2])
                out = float(w.astype(np.float16).astype(np.float64) @ (times * [1, -1]) / (w @ times))
                worst = max(worst, abs(out - ref[r, h * hd]) / bound[r, h * hd])
    report("lower halves", worst=round(worst, 2))
    assert worst > 1.5


def test_tree_attention_captured_graph():
    """One graph over changing trees and lengths; its workspace holds the last replay's partials."""
    torch = torch_cuda()
    a = tree_inputs([9, 30, 1], [800, 300, 77], 16, 4, 2, 64, seed=15, mask="any", behind=6)
    a["slab"] = np.nan_to_num(a["slab"])
    a["table"][:] = np.abs(a["table"]) % a["slab"].shape[0]
    d = {k: dev(a[k]) for k in ("q", "off", "lens", "slab", "table", "mask")}
    d["q"].nan_to_num_()
    a["q"] = d["q"].cpu().numpy()
    out, side = full(a["q"].shape, 7.0, torch.float16), torch.cuda.Stream()
    ws = torch.full((mz.mz_attention_tree_workspace_bytes(a["q"].shape[0], 3, 4, 2, 64) // 4,), float("nan"), device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        tree_run(a, d, ws, out)
    for off, lens in (([0, 9, 39, 40], [800, 300, 77]), ([2, 2, 3, 46], [0, 850, 5]), ([0, 0, 0, 0], [1, 1, 1]), ([0, 20, 20, 46], [31, 9, 700])):
        off, lens = np.array(off, np.int32), np.array(lens, np.int32)
        d["off"].copy_(dev(off))
        d["lens"].copy_(dev(lens))
        out.fill_(7.0)
        g.replay()
        tree_check(a, out, f"replay {off.tolist()}", lens=lens, off=off)


def test_tree_attention_on_two_streams():
    torch = torch_cuda()
    sides = [torch.cuda.Stream() for _ in range(2)]
    args = [tree_inputs([6, 11], [3000 + 500 * i, 900], 64, 8, 2, 128, seed=16 + i) for i in range(2)]
    held = [{k: dev(a[k]) for k in ("q", "off", "lens", "slab", "table", "mask")} for a in args]
    outs = [full(a["q"].shape, 7.0, torch.float16) for a in args]
    wss = [torch.empty(mz.mz_attention_tree_workspace_bytes(a["q"].shape[0], 2, 8, 2, 128), device="cuda", dtype=torch.uint8) for a in args]
    torch.cuda.synchronize()
    for _ in range(4):
        for side, a, d, ws, out in zip(sides, args, held, wss, outs):
            with torch.cuda.stream(side):
                tree_run(a, d, ws, out)
    for a, out in zip(args, outs):
        tree_check(a, out)


# ----------------------------------------------------------------------------- the branch that is taken

def accept_oracle(off, parent, token, choice, lens, m):
    n_seq = len(lens)
    accepted, nxt, len_out, path, ways = np.zeros(n_seq, int), np.full(n_seq, -1), np.zeros(n_seq, int), np.full(m, 7), []
    for b in range(n_seq):
        rows = off[b + 1] - off[b]
        n, way, at = min(rows, 1024), [], 0
        while at is not None and n > 0:
            way.append(at)
            want = choice[off[b] + at]
            nxt[b] = want
            child = [i for i in range(at + 1, n) if (i - 1 if parent is None else parent[off[b] + i]) == at and token[off[b] + i] == want]
            at = child[0] if child and want >= 0 else None
        path[off[b]:off[b + 1]] = way + [-1] * (rows - len(way))
        accepted[b], len_out[b] = len(way), min(max(int(lens[b]), 0), 1 << 30) + len(way)
        ways.append(way)
    return accepted, path, nxt, len_out, ways


def accept_case(counts, lens, C, nkv, hd, layers, seed, tree=True, vocab=3, pad=0, first=0, behind=2, lose=(), tokens=None):
    """vocab: few tokens, so that branches go deep; lose: (sequence, chunk, entry) written over the table."""
    torch = torch_cuda()
    rng = np.random.default_rng(seed)
    off, lens = offsets(counts, first), np.array(lens, np.int32)
    m, dkv, n_seq = int(off[-1]) + behind, nkv * hd, len(counts)
    parent = np.full(m, -1, np.int32)
    for b, n in enumerate(counts):
        parent[off[b]:off[b + 1]] = random_tree(rng, n, 0.1) if n else []
    parent = parent if tree else None
    token, choice = rng.integers(0, vocab, m).astype(np.int32), rng.integers(0, vocab, m).astype(np.int32)
    if tokens:
        token, choice = (np.array(x, np.int32) for x in tokens)
    n_table = (max(max(0, int(x)) for x in lens) + max(counts)) // C + 1
    n_slots = n_seq * n_table + 1
    table = rng.permutation(n_slots)[:n_seq * n_table].reshape(n_seq, n_table).astype(np.int32)
    for s, c, e in lose:
        table[s, c] = e
    stride = n_slots * 2 * C * dkv + pad
    slab = rng.integers(0, 0x7c00, layers * stride).astype(np.uint16).view(np.float16)
    d = [dev(x) if x is not None else None for x in (off, parent, token, choice, lens, table, slab)]
    accepted, nxt, len_out, path = full(n_seq), full(n_seq), full(n_seq), full(m)
    report("accept", counts=list(counts)[:8], lens=list(lens)[:8], C=C, dkv=dkv, layers=layers, seed=seed, tree=tree)
    mz.mz_tree_accept(ptr(d[0]), ptr(d[2]), ptr(d[3]), ptr(d[4]), n_seq, m, ptr(accepted), ptr(path), ptr(nxt), ptr(len_out), stream(),
                      parent_ptr=ptr(d[1]), slab_ptr=ptr(d[6]), n_slots=n_slots, n_layers=layers, layer_bytes=stride * 2,
                      table_ptr=ptr(d[5]), n_table=n_table, chunk_tokens=C, n_kv=nkv, head_dim=hd)
    torch.cuda.synchronize()
    ref = accept_oracle(off, parent, token, choice, lens, m)
    for got, want, what in zip((accepted, path, nxt, len_out), ref, ("accepted", "path", "next", "len_out")):
        assert np.array_equal(got.cpu().numpy(), want), what
    want = slab.copy().view(np.uint16)
    for layer in range(layers):
        part = want[layer * stride:layer * stride + n_slots * 2 * C * dkv].reshape(n_slots, 2, C * dkv)
        before = part.copy()
        for b, way in enumerate(ref[4]):
            start = min(max(int(lens[b]), 0), 1 << 30)
            for i, node in enumerate(way):
                (x, p), (y, r) = (((start + j) // C, (start + j) % C) for j in (node, i))
                if x >= n_table or y >= n_table or not (0 <= table[b, x] < n_slots and 0 <= table[b, y] < n_slots):
                    continue
                x, y = table[b, x], table[b, y]
                part[y, 0].reshape(C, dkv)[r] = before[x, 0].reshape(C, dkv)[p]
                part[y, 1].reshape(dkv, C)[:, r] = before[x, 1].reshape(dkv, C)[:, p]
    assert np.array_equal(d[6].cpu().numpy().view(np.uint16), want), "slab"
    return ref


@pytest.mark.parametrize("n", [1, 2, 3, 31, 64, 65, 130, 300])
@pytest.mark.parametrize("C,nkv,hd,layers", [(8, 1, 32, 1), (16, 2, 64, 3), (64, 8, 128, 2)])
def test_accept_trees(n, C, nkv, hd, layers):
    deep = 0
    for seed in range(3):
        got = accept_case([n, 0, n // 2 + 1], [5, 9, 30], C, nkv, hd, layers, seed=n + seed, vocab=2, pad=8 * seed)
        deep = max(deep, int(got[0].max()))
    assert n < 31 or deep >= 3


def test_accept_chains():
    accept_case([12, 1, 40], [7, 0, 100], 16, 2, 64, 2, seed=1, tree=False, vocab=1)
    accept_case([12, 1, 40], [7, 0, 100], 16, 2, 64, 2, seed=2, tree=False, vocab=2, first=3)
    accept_case([1100], [7], 64, 1, 32, 1, seed=3, tree=False, vocab=1)


@pytest.mark.parametrize("n,miss", [(1023, None), (1024, None), (1025, None), (2500, None), (2500, 1022), (2500, 1023), (2500, 1024), (5000, 3000)])
def test_accept_chains_of_more_nodes_than_a_call_takes(n, miss):
    """A call takes the first 1024 nodes, calls on the rest what follows: together the whole branch; miss: the node whose
    choice is not the next one's token."""
    torch = torch_cuda()
    rng = np.random.default_rng(n)
    token = rng.integers(0, 1000, n).astype(np.int32)
    choice = np.append(token[1:], 5).astype(np.int32)
    if miss is not None:
        choice[miss] = (choice[miss] + 1) % 1000
    whole = n if miss is None else miss + 1
    d_token, d_choice, lens, at, total = dev(token), dev(choice), dev(np.array([77], np.int32)), 0, 0
    while True:
        report("accept", n=n, miss=miss, at=at)
        accepted, path, nxt, len_out, off = full(1), full(n), full(1), full(1), dev(np.array([at, n], np.int32))
        mz.mz_tree_accept(ptr(off), ptr(d_token), ptr(d_choice), ptr(lens), 1, n, ptr(accepted), ptr(path), ptr(nxt), ptr(len_out), stream())
        torch.cuda.synchronize()
        count = min(whole - at, 1024)
        want = np.full(n, -1)
        want[:at] = 7      # rows before the chain are left as they are
        want[at:at + count] = np.arange(count)
        assert accepted.tolist() == [count] and nxt.tolist() == [choice[at + count - 1]] and len_out.tolist() == [77 + at + count]
        assert np.array_equal(path.cpu().numpy(), want)
        total, lens, at = total + count, len_out, at + count
        if at == n or nxt.item() != token[at]:
            break
    assert total == whole


def test_accept_moves_a_long_branch():
    """A branch of more places than a thread holds at once, every place moved by one."""
    n = 40
    torch_cuda()
    rng = np.random.default_rng(4)
    token, choice = np.arange(n) + 5, np.arange(n) + 6
    token[1] = 999      # node 1 is not taken: 0 -> 2 -> 3 -> ...
    choice[0] = token[2]
    del rng
    off, lens = np.array([0, n], np.int32), np.array([13], np.int32)
    parent = np.array([-1, 0, 0] + list(range(2, n - 1)), np.int32)
    torch = torch_cuda()
    C, dkv, n_slots = 8, 64, 8
    slab = np.random.default_rng(5).integers(0, 0x7c00, (n_slots, 2, dkv * C)).astype(np.uint16)
    d = [dev(x) for x in (off, parent, token.astype(np.int32), choice.astype(np.int32), lens, np.arange(8, dtype=np.int32)[None], slab.view(np.float16))]
    accepted, nxt, len_out, path = full(1), full(1), full(1), full(n)
    mz.mz_tree_accept(ptr(d[0]), ptr(d[2]), ptr(d[3]), ptr(d[4]), 1, n, ptr(accepted), ptr(path), ptr(nxt), ptr(len_out), stream(),
                      parent_ptr=ptr(d[1]), slab_ptr=ptr(d[6]), n_slots=n_slots, n_layers=1, table_ptr=ptr(d[5]), n_table=8, chunk_tokens=C,
                      n_kv=1, head_dim=64)
    torch.cuda.synchronize()
    assert accepted.item() == n - 1 and len_out.item() == 13 + n - 1 and nxt.item() == n + 5
    keys = slab[:, 0].reshape(n_slots * C, dkv).copy()
    keys[14:14 + n - 2] = keys[15:15 + n - 2].copy()
    values = slab[:, 1].reshape(n_slots, dkv, C).transpose(0, 2, 1).reshape(-1, dkv).copy()
    values[14:14 + n - 2] = values[15:15 + n - 2].copy()
    got = d[6].cpu().numpy().view(np.uint16).reshape(n_slots, 2, -1)
    assert np.array_equal(got[:, 0].reshape(-1, dkv), keys)
    assert np.array_equal(got[:, 1].reshape(n_slots, dkv, C).transpose(0, 2, 1).reshape(-1, dkv), values)


def test_accept_edges():
    accept_case([5, 5], [0, -4], 8, 1, 64, 1, seed=6, tokens=([1, 1, 1, 1, -1, 1, 2, 2, 2, 2, 0, 0], [1, 1, 1, 1, -1, -1, -1, 2, 2, 2, 0, 0]))
    accept_case([20, 30], [50, 3], 8, 1, 32, 2, seed=7, vocab=1, lose=((0, 7, -1), (1, 0, 1 << 20), (1, 2, -5)))
    accept_case([3] * 300, list(range(300)), 16, 1, 32, 1, seed=8, vocab=2)


def test_accept_without_a_cache():
    torch = torch_cuda()
    off, token, choice, lens = (dev(np.array(x, np.int32)) for x in ([0, 4], [9, 5, 6, 7], [5, 6, 8, 1], [(1 << 31) - 1]))
    accepted, path, nxt, len_out = full(1), full(4), full(1), full(1)
    mz.mz_tree_accept(ptr(off), ptr(token), ptr(choice), ptr(lens), 1, 4, ptr(accepted), ptr(path), ptr(nxt), ptr(len_out), stream())
    torch.cuda.synchronize()
    assert accepted.tolist() == [3] and path.tolist() == [0, 1, 2, -1] and nxt.tolist() == [8] and len_out.tolist() == [(1 << 30) + 3]


def test_accept_past_the_table():
    """Places beyond the table are not moved, nothing behind it is touched."""
    torch = torch_cuda()
    off, token, choice, lens, table, parent = (dev(np.array(x, np.int32)) for x in
                                               ([0, 6], [0] * 6, [0] * 6, [13], [[1, 0]], [-1, 5, 0, 0, 2, 4]))
    slab = torch.randn(3, 2 * 8 * 32, device="cuda").half()
    old = slab.clone()
    accepted, path, nxt, len_out = full(1), full(6), full(1), full(1)
    mz.mz_tree_accept(ptr(off), ptr(token), ptr(choice), ptr(lens), 1, 6, ptr(accepted), ptr(path), ptr(nxt), ptr(len_out), stream(),
                      parent_ptr=ptr(parent), slab_ptr=ptr(slab), n_slots=2, n_layers=1, table_ptr=ptr(table), n_table=2, chunk_tokens=8,
                      n_kv=1, head_dim=32)
    torch.cuda.synchronize()
    assert path.tolist() == [0, 2, 4, 5, -1, -1]      # 15 -> 14 moves; 17 and 18 lie behind the table
    old[0, :256].view(8, 32)[6] = old[0, :256].view(8, 32)[7]
    old[0, 256:].view(32, 8)[:, 6] = old[0, 256:].view(32, 8)[:, 7]
    assert torch.equal(slab, old)


# ----------------------------------------------------------------------------- pages

def pages_oracle(table, src, keep, room, n_slots, limit, C):
    """(table, info, copies)."""
    n_seq, wide = table.shape
    top = wide * C
    src = list(range(n_seq)) if src is None else [int(x) for x in src]
    keep = [min(max(int(k), 0), top) if 0 <= s < n_seq else 0 for k, s in zip(keep, src)]
    end = [min(k + (0 if room is None else max(int(room[i]), 0)), top) for i, k in enumerate(keep)]
    new, holders = np.full(table.shape, -1), {}
    for b in range(n_seq):
        for c in range(-(-keep[b] // C)):
            e = int(table[src[b], c])
            if 0 <= e < n_slots:
                new[b, c] = e
                holders.setdefault(e, []).append((b, c))
    forks = set()
    for e, who in holders.items():
        if len(who) == 1:
            continue
        writing = [(b, c) for b, c in who if end[b] > keep[b] and keep[b] % C and c == keep[b] // C]
        stays = min(writing, key=lambda w: (src[w[0]] != w[0], w[0])) if len(writing) == len(who) else None
        forks |= {w for w in writing if w != stays}
    moves = [e for e in sorted(holders) if e >= limit and any(w not in forks for w in holders[e])]
    wants = [("move", e, 0) for e in moves]
    for b in range(n_seq):
        for c in range(wide):
            if (b, c) in forks:
                wants.append(("fork", b, c))
            elif keep[b] // C <= c < -(-end[b] // C) and end[b] > keep[b] and new[b, c] < 0:
                wants.append(("new", b, c))
    free = [e for e in range(limit) if e not in holders]
    held = len(holders) + len(wants) - len(moves)
    if len(wants) > len(free):
        return table.copy(), [len(wants) - len(free), held, 0, 0], []
    to = dict(zip(wants, free))
    copies = [(e, to["move", e, 0], C, 0) for e in moves]
    out = np.vectorize(lambda e: to.get(("move", int(e), 0), int(e)))(new)
    for kind, b, c in wants:
        if kind == "fork":
            copies.append((int(new[b, c]), to[kind, b, c], keep[b] % C, 0))
        if kind != "move":
            out[b, c] = to[kind, b, c]
    return out, [0, held, len(copies), 0], copies


def pages_run(table, src, keep, room, n_slots, limit, C, in_place=False):
    torch = torch_cuda()
    n_seq, wide = table.shape
    d = [None if x is None else dev(np.asarray(x, np.int32)) for x in (table, src, keep, room)]
    out = d[0] if in_place else full(table.shape)
    most = n_seq + n_slots - (limit or n_slots)
    copies, info = full((most + 1, 4)), full(4)
    need = mz.mz_kv_pages_workspace_bytes(n_seq, wide, n_slots)
    ws = torch.full((need // 4,), -1, device="cuda", dtype=torch.int32)
    mz.mz_kv_pages(ptr(d[0]), ptr(out), n_seq, wide, n_slots, C, ptr(d[2]), ptr(copies), ptr(info), ptr(ws), need, stream(),
                   src_ptr=ptr(d[1]), room_ptr=ptr(d[3]), slot_limit=limit)
    torch.cuda.synchronize()
    assert (copies[-1] == 7).all()
    return out.cpu().numpy(), info.tolist(), copies.cpu().numpy(), (copies, info)


def pages_case(table, src, keep, room, n_slots, limit, C):
    table = np.asarray(table, np.int32)
    report("pages", n_seq=table.shape[0], wide=table.shape[1], n_slots=n_slots, limit=limit, C=C)
    want, info, copies = pages_oracle(table, src, keep, room, n_slots, limit or n_slots, C)
    for in_place in (False, True):
        got, ginfo, gcopies, _ = pages_run(table, src, keep, room, n_slots, limit, C, in_place)
        assert ginfo == info, (ginfo, info)
        assert np.array_equal(got, want), (got, want)
        assert [tuple(x) for x in gcopies[:len(copies)]] == copies
        assert (gcopies[len(copies):] == 7).all(), "more entries than copies"
    return want, info, copies


def pages_inputs(rng, n_seq, wide, n_slots, C):
    """Tables with rows of shared chunks, rows without any and entries that are no slots."""
    table = np.full((n_seq, wide), -1, np.int64)
    free = list(rng.permutation(n_slots))
    for b in range(n_seq):
        n = int(rng.integers(0, wide + 1))
        shared = int(rng.integers(0, n + 1)) if b and rng.random() < 0.5 else 0
        other = int(rng.integers(0, b)) if b else 0
        for c in range(n):
            if c < shared and table[other, c] >= 0:
                table[b, c] = table[other, c]
            elif free and rng.random() < 0.95:
                table[b, c] = free.pop()
            elif rng.random() < 0.5:
                table[b, c] = rng.choice([-5, n_slots, 1 << 30])
    src = [b if rng.random() < 0.5 else int(rng.integers(-1, n_seq + 1)) for b in range(n_seq)]
    top = wide * C
    keep = [int(rng.choice([0, rng.integers(-3, top + 5), rng.integers(0, wide + 1) * C])) for _ in range(n_seq)]
    room = [int(rng.choice([0, 1, rng.integers(-3, 3 * C)])) for _ in range(n_seq)]
    return table, src, keep, room


@pytest.mark.parametrize("seed", range(12))
def test_pages_random(seed):
    rng = np.random.default_rng(seed)
    C = int(rng.choice([8, 16, 64]))
    n_seq, wide = int(rng.integers(1, 30)), int(rng.integers(1, 20))
    n_slots = int(rng.integers(1, 3 * n_seq * wide + 2))
    table, src, keep, room = pages_inputs(rng, n_seq, wide, n_slots, C)
    pages_case(table, src, keep, room, n_slots, 0, C)
    pages_case(table, src, keep, room, n_slots, int(rng.integers(1, n_slots + 1)), C)
    pages_case(table, None, keep, room, n_slots, max(1, n_slots - n_slots // 4), C)
    pages_case(table, src, keep, None, n_slots, 0, C)


@pytest.mark.parametrize("n_seq,wide,n_slots", [(1024, 20, 8192), (1025, 7, 8000), (64, 320, 8192), (64, 321, 8192), (64, 300, 8193), (4, 5121, 8000), (1, 1, 1), (3, 5000, 20000), (1500, 7, 9000), (70, 300, 40000), (1100, 20, 16384)])
def test_pages_sizes(n_seq, wide, n_slots):
    rng = np.random.default_rng(n_seq)
    table, src, keep, room = pages_inputs(rng, n_seq, wide, n_slots, 8)
    pages_case(table, src, keep, room, n_slots, 0, 8)
    pages_case(table, src, keep, room, n_slots, n_slots * 3 // 4, 8)
    pages_case(table, None, [1 << 30] * n_seq, None, n_slots, 0, 8)
    pages_case(table, None, [0] * n_seq, None, n_slots, 0, 8)


@pytest.mark.parametrize("n_seq,wide,n_slots", [(16, 1280, 8192), (16, 1281, 8192), (1, 20480, 8000), (1, 20481, 8000), (256, 80, 8192), (256, 81, 8192),
                                                (1024, 16, 700), (1025, 16, 700)])
def test_pages_on_both_sides_of_one_workgroup(n_seq, wide, n_slots):
    """Tables that one workgroup takes and that it leaves to several launches; rows that all write the chunk that they share."""
    rng = np.random.default_rng(n_seq + wide)
    table, src, keep, room = pages_inputs(rng, n_seq, wide, n_slots, 8)
    pages_case(table, src, keep, room, n_slots, 0, 8)
    pages_case(table, None, keep, room, n_slots, n_slots * 3 // 4, 8)
    pages_case(table, [n_seq - 1] * n_seq, [19] * n_seq, [3] * n_seq, n_slots, 0, 8)


def test_pages_forks_and_beams():
    C, t = 8, [[3, 4, -1], [5, -1, -1], [6, 7, -1], [-1, -1, -1]]
    # a fork of a chunk that both write: the row that stays keeps it
    assert pages_case(t, [0, 0, 2, -1], [11, 11, 9, 0], [1, 1, 1, 20], 20, 0, C)[2] == [(4, 0, 3, 0)]
    # beams change places, nobody stays: the lowest keeps the chunk
    assert pages_case(t, [2, 2, 0, 0], [11, 11, 9, 9], [1] * 4, 20, 0, C)[2] == [(7, 0, 3, 0), (4, 1, 1, 0)]
    # one of the two only reads: the one that writes copies; no room: none does
    assert pages_case(t, [0, 0, 2, -1], [11, 11, 9, 0], [0, 1, 1, 0], 20, 0, C)[2] == [(4, 0, 3, 0)]
    assert pages_case(t, [0, 0, 2, -1], [11, 11, 9, 0], None, 20, 0, C)[2] == []
    # whole chunks are shared without a copy
    assert pages_case(t, [0, 0, 0, 0], [16] * 4, [1] * 4, 20, 0, C)[2] == []
    # the slots that are freed serve in the same call; one is missing: nothing changes
    assert pages_case(t, [-1, -1, 2, -1], [0, 0, 9, 0], [24, 0, 1, 0], 8, 3, C)[1][0] > 0
    assert pages_case(t, [-1, -1, 2, -1], [0, 0, 9, 0], [24, 24, 1, 0], 8, 0, C)[1][:2] == [0, 8]
    assert pages_case(t, [-1, -1, 2, -1], [0, 0, 9, 0], [24, 25, 9, 0], 8, 0, C)[1][:2] == [1, 9]


def copy_case(copies, n, C, nkv, hd, layers, n_slots, pad=0, most=None):
    torch = torch_cuda()
    rng = np.random.default_rng(C + hd)
    dkv, stride = nkv * hd, n_slots * 2 * C * nkv * hd + pad
    slab = rng.integers(0, 0x7c00, layers * stride).astype(np.uint16)
    d, d_copies, d_n = dev(slab.view(np.float16)), dev(np.array(copies, np.int32).reshape(-1, 4)), dev(np.array([n], np.int32))
    mz.mz_kv_copy(ptr(d_copies), ptr(d_n), len(copies) if most is None else most, ptr(d), n_slots, layers, stride * 2, C, nkv, hd, stream())
    torch.cuda.synchronize()
    for layer in range(layers):
        part = slab[layer * stride:layer * stride + n_slots * 2 * C * dkv].reshape(n_slots, 2, C * dkv)
        for x, y, t, _ in copies[:min(max(n, 0), len(copies) if most is None else most)]:
            if 0 <= x < n_slots and 0 <= y < n_slots and x != y:
                t = min(max(t, 0), C)
                part[y, 0].reshape(C, dkv)[:t] = part[x, 0].reshape(C, dkv)[:t]
                part[y, 1].reshape(dkv, C)[:, :t] = part[x, 1].reshape(dkv, C)[:, :t]
    assert np.array_equal(d.cpu().numpy().view(np.uint16), slab)


@pytest.mark.parametrize("C,nkv,hd,layers", [(8, 1, 32, 1), (16, 2, 64, 3), (64, 3, 32, 2), (256, 8, 128, 2)])
def test_copy(C, nkv, hd, layers):
    tokens = sorted({0, 1, 7, 8, 9, C // 2 + 1, C - 1, C, C + 9, -3})
    n_slots = len(tokens) + 3
    copies = [(i % 2, i + 3, t, 0) for i, t in enumerate(tokens)]
    copy_case(copies, len(copies), C, nkv, hd, layers, n_slots, pad=16)
    copy_case(copies, len(copies) - 2, C, nkv, hd, layers, n_slots)
    copy_case(copies, 1 << 30, C, nkv, hd, layers, n_slots, most=3)
    copy_case(copies, -1, C, nkv, hd, layers, n_slots)
    copy_case([(0, 0, C, 0), (-1, 2, C, 0), (1, n_slots, C, 0), (1, 2, C, 0)], 4, C, nkv, hd, layers, n_slots)


def test_copy_far_slots():
    """Slots and layers past 2^32 bytes."""
    torch = torch_cuda()
    C, nkv, hd = 64, 2, 128
    n_slots = (1 << 32) // (C * nkv * hd * 4) + 3
    slab = torch.zeros(2, n_slots, 2 * C * nkv * hd, device="cuda", dtype=torch.float16)
    slab[:, 1].normal_()
    slab[:, n_slots - 1].normal_()
    want = slab[:, [1, n_slots - 1]].clone()
    copies, n = dev(np.array([[1, n_slots - 2, C, 0], [n_slots - 1, 2, C, 0]], np.int32)), dev(np.array([2], np.int32))
    mz.mz_kv_copy(ptr(copies), ptr(n), 2, ptr(slab), n_slots, 2, slab.stride(0) * 2, C, nkv, hd, stream())
    torch.cuda.synchronize()
    assert torch.equal(slab[:, [n_slots - 2, 2]], want)


# ----------------------------------------------------------------------------- together

def test_a_step_that_checks_drafted_trees():
    """Pages, copies, rows, appending, attention and the branch in one graph, replayed over forks, trees and lengths that
    change, against a cache that is kept token by token on the host."""
    torch = torch_cuda()
    rng = np.random.default_rng(1)
    layers, nq, nkv, hd, C, n_seq, m, n_table, n_slots, n_rope = 2, 8, 2, 64, 16, 4, 40, 8, 40, 200
    dq, dkv, words, limit = nq * hd, nkv * hd, 1, 34
    rope = rope_table(n_rope, hd)
    z = lambda *shape, dtype=torch.int32: torch.zeros(shape, device="cuda", dtype=dtype)  # noqa: E731
    table, src, keep, room, info = full((n_seq, n_table), -1), z(n_seq), z(n_seq), z(n_seq), z(4)
    copies = z(n_seq + n_slots - limit, 4)
    off, parent, token, choice, lens = z(n_seq + 1), z(m), z(m), z(m), z(n_seq)
    seq, place, rpos, mask = z(m), z(m), z(m), z(m, words)
    accepted, path, nxt, len_out = z(n_seq), z(m), z(n_seq), z(n_seq)
    qkv, q_rot, out = z(layers, m, dq + 2 * dkv, dtype=torch.float32), z(layers, m, dq, dtype=torch.float16), z(layers, m, dq, dtype=torch.float16)
    slab, d_rope = z(layers, n_slots, 2 * C * dkv, dtype=torch.float16), dev(rope)
    pws = z(mz.mz_kv_pages_workspace_bytes(n_seq, n_table, n_slots), dtype=torch.uint8)
    aws = z(mz.mz_attention_tree_workspace_bytes(m, n_seq, nq, nkv, hd), dtype=torch.uint8)
    slab.fill_(float("nan"))

    def step():
        mz.mz_kv_pages(ptr(table), ptr(table), n_seq, n_table, n_slots, C, ptr(keep), ptr(copies), ptr(info), ptr(pws), pws.numel(), stream(),
                       src_ptr=ptr(src), room_ptr=ptr(room), slot_limit=limit)
        mz.mz_kv_copy(ptr(copies), ptr(info) + 8, copies.shape[0], ptr(slab), n_slots, layers, slab.stride(0) * 2, C, nkv, hd, stream())
        mz.mz_tree_plan(ptr(off), ptr(lens), n_seq, m, stream(), parent_ptr=ptr(parent), seq_ptr=ptr(seq), place_ptr=ptr(place),
                        rope_pos_ptr=ptr(rpos), mask_ptr=ptr(mask), mask_words=words)
        for x in range(layers):
            base = ptr(qkv[x])
            mz.mz_kv_append_axes(m, base + dq * 4, base + (dq + dkv) * 4, ptr(seq), ptr(place), ptr(rpos), 1, [0] * (hd // 2), ptr(d_rope), n_rope,
                                 ptr(slab[x]), n_slots, ptr(table), n_seq, n_table, C, nkv, hd, stream(), q_ptr=base, n_q=nq,
                                 q_out_ptr=ptr(q_rot[x]), k_stride=dq + 2 * dkv, v_stride=dq + 2 * dkv, q_stride=dq + 2 * dkv)
            mz.mz_attention_tree(ptr(q_rot[x]), m, ptr(off), ptr(lens), n_seq, ptr(slab[x]), n_slots, ptr(table), n_table, C, nq, nkv, hd,
                                 ptr(aws), aws.numel(), ptr(out[x]), stream(), mask_ptr=ptr(mask), mask_words=words)
        mz.mz_tree_accept(ptr(off), ptr(token), ptr(choice), ptr(lens), n_seq, m, ptr(accepted), ptr(path), ptr(nxt), ptr(len_out), stream(),
                          parent_ptr=ptr(parent), slab_ptr=ptr(slab), n_slots=n_slots, n_layers=layers, layer_bytes=slab.stride(0) * 2,
                          table_ptr=ptr(table), n_table=n_table, chunk_tokens=C, n_kv=nkv, head_dim=hd)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step()
    caches = [[np.zeros((0, 2 * dkv), np.float16)] * n_seq for _ in range(layers)]      # keys and values of every sequence
    now = [0] * n_seq
    deep = forked = 0
    for turn in range(12):
        sources = [b if turn < 2 or rng.random() < 0.6 else int(rng.integers(-1, n_seq)) for b in range(n_seq)]
        kept = [now[s] if s >= 0 else 0 for s in sources]
        kept = [int(rng.integers(0, k + 1)) if rng.random() < 0.2 else min(k, n_table * C - 20) for k in kept]
        counts = [int(rng.integers(0, 11)) if b else 10 for b in range(n_seq)]
        h_off = offsets(counts)
        h_parent, h_token, h_choice = np.full(m, -1, np.int32), rng.integers(0, 2, m).astype(np.int32), rng.integers(0, 2, m).astype(np.int32)
        for b, n in enumerate(counts):
            h_parent[h_off[b]:h_off[b + 1]] = random_tree(rng, n)
        h_qkv = rng.standard_normal((layers, m, dq + 2 * dkv)).astype(np.float32)
        for x, v in ((src, sources), (keep, kept), (lens, kept), (room, counts), (off, h_off), (parent, h_parent), (token, h_token), (choice, h_choice),
                     (qkv, h_qkv)):
            x.copy_(dev(np.asarray(v, np.float32 if x is qkv else np.int32)))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert info.tolist()[0] == 0, "slots are missing"
        forked += info.tolist()[2]
        h_table = table.cpu().numpy()
        plan = plan_oracle(h_off, h_parent, np.array(kept), m, words)
        ways = accept_oracle(h_off, h_parent, h_token, h_choice, np.array(kept), m)
        assert accepted.tolist() == ways[0].tolist() and len_out.tolist() == ways[3].tolist() and nxt.tolist() == ways[2].tolist()
        deep = max(deep, int(ways[0].max()))
        for x in range(layers):
            halves = slab[x].cpu().numpy().reshape(n_slots, 2, -1)
            got_q, got = q_rot[x].cpu().numpy(), out[x]
            old, caches[x] = caches[x], []
            rows = [np.zeros((0, 2 * dkv), np.float16)] * n_seq
            for b in range(n_seq):
                # keys of the branch as the append leaves them: read from the slab before the move would need another copy, so turn them here
                part = []
                for r in range(h_off[b], h_off[b + 1]):
                    a = h_qkv[x, r, dq:dq + dkv].reshape(nkv, hd).astype(np.float64)
                    c, s = rope[plan[2][r], :, 0].astype(np.float64), rope[plan[2][r], :, 1].astype(np.float64)
                    y = np.concatenate([a[:, :hd // 2] * c - a[:, hd // 2:] * s, a[:, hd // 2:] * c + a[:, :hd // 2] * s], 1)
                    part.append(np.concatenate([y.reshape(-1), h_qkv[x, r, dq + dkv:].astype(np.float16).astype(np.float64)]))
                rows[b] = np.array(part).reshape(-1, 2 * dkv)
                before = old[sources[b]][:kept[b]].astype(np.float64) if sources[b] >= 0 else np.zeros((0, 2 * dkv))
                # the rows' outputs: the keys are at most half a step of f16 off, which moves a score by at most 2 U16 |q| |k|
                for i in range(counts[b]):
                    r = h_off[b] + i
                    seen = [j for j in range(counts[b]) if plan[3][r, 0] >> j & 1]
                    kv = np.concatenate([before, rows[b][seen]])
                    for h in range(nq):
                        kk, vv = kv[:, h // 4 * hd:][:, :hd], kv[:, dkv + h // 4 * hd:][:, :hd]
                        q = got_q[r, h * hd:(h + 1) * hd].astype(np.float64)
                        w = kk @ q / 8
                        p = np.exp(w - w.max())
                        p /= p.sum()
                        e = 2 * U16 * (np.abs(kk) @ np.abs(q)).max() / 8 + 2.0 ** -18
                        ref, size = p @ vv, p @ np.abs(vv)
                        diff = np.abs(got[r, h * hd:(h + 1) * hd].double().cpu().numpy() - ref)
                        assert (diff <= 2.1 * e * size + U16 * np.abs(ref) + TINY16).all(), (turn, x, b, i, h)
                after = np.concatenate([before, rows[b][ways[4][b]]]) if ways[4][b] else before
                # what the cache holds now, through the table
                pos = np.arange(after.shape[0])
                at = h_table[b, pos // C]
                assert (at >= 0).all() and (at < limit).all()
                held = np.concatenate([halves[at, 0].reshape(-1, C, dkv)[np.arange(pos.size), pos % C],
                                       halves[at, 1].reshape(-1, dkv, C)[np.arange(pos.size), :, pos % C]], 1) if pos.size else np.zeros((0, 2 * dkv), np.float16)
                assert (np.abs(held.astype(np.float64) - after) <= U16 * np.abs(after) * (1 + U16) + TINY16 + 8 * U32).all(), (turn, x, b)
                caches[x].append(held)
        now = [int(v) for v in ways[3]]
    assert deep >= 3 and forked >= 3
