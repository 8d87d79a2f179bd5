"""The calls that carry a decode step of many sequences -- the append to the
chunked caches, the attention over them, the adapters beside a projection and
the rules on the logits -- against plain implementations in 64 bits.

Roundings: u16 = 2^-11 is half a step of f16 relative to the value (2^-25
below its normal range), u32 = 2^-24 half a step of fp32.
"""

import numpy as np
import pytest

from paper_2609_01338_amd import mz
from gpu_util import report, stream, torch_cuda

pytestmark = pytest.mark.gpu

U16, U32, TINY16 = 2.0 ** -11, 2.0 ** -24, 2.0 ** -25


def dev(a):
    return torch_cuda().from_numpy(np.ascontiguousarray(a)).cuda()


def close(got, ref, bound, what):
    """got (device or host) within bound of ref everywhere; NaN and infinities at the same places."""
    got = got.double().cpu().numpy() if hasattr(got, "cpu") else np.asarray(got, np.float64)
    ref, bound = np.broadcast_arrays(np.asarray(ref, np.float64), np.asarray(bound, np.float64))
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), what + ": NaN"
    assert np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)]), what + ": infinities"
    err = np.abs(got[fine] - ref[fine])
    worst = float((err / np.maximum(bound[fine], 1e-300)).max()) if err.size else 0.0
    report("  " + what, worst_of_bound=round(worst, 4), max_err=float(err.max()) if err.size else 0.0)
    assert np.all(err <= bound[fine]), what


def rope_table(n, hd, theta=1e4):
    a = np.arange(n)[:, None] * theta ** (-2.0 * np.arange(hd // 2) / hd)
    return np.stack([np.cos(a), np.sin(a)], 2).astype(np.float32)


# ----------------------------------------------------------------------------- append

def append_oracle(k, v, q, seq, pos, rope, slab, table, C, nkv, hd):
    """What the rows leave: (slab, its bound, q, its bound, rows of q that are written)."""
    m, n_slots = len(seq), slab.shape[0]
    dkv, h2 = nkv * hd, hd // 2

    def turn(x, p):
        c, s = rope[p, :, 0].astype(np.float64), rope[p, :, 1].astype(np.float64)
        a, b = x[:, :h2], x[:, h2:]
        y = np.concatenate([a * c - b * s, b * c + a * s], 1)
        part = np.concatenate([np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)], 1)
        # two fp32 roundings, then one to f16
        return y, U16 * np.abs(y) + TINY16 + 2 * U32 * part * (1 + U16)

    out, bound = slab.astype(np.float64), np.zeros(slab.shape)
    kh, vh = out[:, :C * dkv].reshape(n_slots, C, nkv, hd), out[:, C * dkv:].reshape(n_slots, dkv, C)
    kb = bound[:, :C * dkv].reshape(n_slots, C, nkv, hd)
    qo, qb, wrote = None, None, np.zeros(m, bool)
    if q is not None:
        qo, qb = np.zeros(q.shape), np.zeros(q.shape)
    for r in range(m):
        s, p = int(seq[r]), int(pos[r])
        if not (0 <= s < table.shape[0] and 0 <= p < rope.shape[0] and p // C < table.shape[1]):
            continue
        if q is not None:
            y, b = turn(q[r].reshape(-1, hd).astype(np.float64), p)
            qo[r], qb[r], wrote[r] = y.reshape(-1), b.reshape(-1), True
        slot = int(table[s, p // C])
        if 0 <= slot < n_slots:
            kh[slot, p % C], kb[slot, p % C] = turn(k[r].reshape(nkv, hd).astype(np.float64), p)
            vh[slot, :, p % C] = v[r].astype(np.float16).astype(np.float64)
    return out, bound, qo, qb, wrote


def append_run(k, v, q, seq, pos, rope, slab, table, C, nkv, hd, f32, fused, st=None):
    torch = torch_cuda()
    m, dkv = len(seq), nkv * hd
    dt, size = (np.float32, 4) if f32 else (np.float16, 2)
    d_slab, d_rope, d_seq, d_pos, d_table = dev(slab), dev(rope), dev(seq), dev(pos), dev(table)
    nq = 0 if q is None else q.shape[1] // hd
    q_out = torch.full((m, max(nq, 1) * hd), 7.0, device="cuda", dtype=torch.float16)
    kw = {}
    if fused:      # one buffer of rows, as a projection leaves them, with a tail behind each row
        parts = ([q] if q is not None else []) + [k, v, np.full((m, 16), np.nan)]
        rows = dev(np.concatenate(parts, 1).astype(dt))
        base = rows.data_ptr()
        kp, vp = base + nq * hd * size, base + (nq * hd + dkv) * size
        kw = dict(k_stride=rows.shape[1], v_stride=rows.shape[1], q_stride=rows.shape[1])
        if q is not None:
            kw.update(q_ptr=base, n_q=nq, q_out_ptr=q_out.data_ptr())
    else:
        dk, dv = dev(k.astype(dt)), dev(v.astype(dt))
        kp, vp = dk.data_ptr(), dv.data_ptr()
        if q is not None:
            dq = dev(q.astype(dt))
            kw.update(q_ptr=dq.data_ptr(), n_q=nq, q_out_ptr=q_out.data_ptr())
    mz.mz_kv_append(m, kp, vp, d_seq.data_ptr(), d_pos.data_ptr(), d_rope.data_ptr(), rope.shape[0], d_slab.data_ptr(),
                    slab.shape[0], d_table.data_ptr(), table.shape[0], table.shape[1], C, nkv, hd,
                    stream() if st is None else st, f32=f32, **kw)
    torch.cuda.synchronize()
    return d_slab, q_out


def append_case(spans, C, nq, nkv, hd, f32, seed, shuffle=False, extra=(), fused=True, bad_slots=()):
    """spans: (first position, rows) per sequence; extra: (seq, pos) rows that must write nothing;
    bad_slots: (sequence, chunk, entry) written over the table."""
    rng = np.random.default_rng(seed)
    rows = [(s, p + i) for s, (p, n) in enumerate(spans) for i in range(n)] + list(extra)
    if shuffle:
        rng.shuffle(rows)
    seq, pos = (np.array([r[i] for r in rows], np.int32) for i in (0, 1))
    m, n_table = len(rows), max(p + n for p, n in spans) // C + 1
    n_slots = len(spans) * n_table + 3
    table = rng.permutation(n_slots)[:len(spans) * n_table].reshape(len(spans), n_table).astype(np.int32)
    for s, c, e in bad_slots:
        table[s, c] = e
    rope = rope_table(max(p + n for p, n in spans), hd)
    dt = np.float32 if f32 else np.float16
    draw = lambda h: rng.standard_normal((m, h * hd)).astype(dt)  # noqa: E731
    q, k, v = (draw(nq) if nq else None), draw(nkv), draw(nkv)
    for r, (s, p) in enumerate(rows):      # rows that write nothing hold no numbers
        if (s, p) in extra:
            k[r], v[r] = np.nan, np.inf
    slab = rng.standard_normal((n_slots, 2 * C * nkv * hd)).astype(np.float16)
    report("append", spans=spans, C=C, nq=nq, nkv=nkv, hd=hd, f32=f32, m=m, seed=seed)
    got, q_got = append_run(k, v, q, seq, pos, rope, slab, table, C, nkv, hd, f32, fused)
    ref, bound, q_ref, q_bound, wrote = append_oracle(k, v, q, seq, pos, rope, slab, table, C, nkv, hd)
    close(got, ref, bound, "slab")
    if nq:
        close(q_got[dev(wrote)], q_ref[wrote], q_bound[wrote], "q")
        assert bool((q_got[dev(~wrote)] == 7).all()), "a row that writes nothing"


@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 64), (32, 8, 64), (12, 2, 128), (8, 8, 128), (0, 1, 64), (5, 1, 32), (3, 3, 32)])
@pytest.mark.parametrize("f32", [True, False])
def test_append_one_row_each(nq, nkv, hd, f32):
    append_case([(p, 1) for p in (0, 1, 15, 16, 77, 255, 256, 300)], 16, nq, nkv, hd, f32, seed=nq + hd)


@pytest.mark.parametrize("C", [8, 16, 64, 256])
@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("spans", [[(0, 1)], [(0, 64)], [(0, 200)], [(3, 71), (0, 8), (250, 140), (9, 7)],
                                   [(511, 1), (8, 57), (0, 63), (1, 129)]])
def test_append_prompts(spans, C, f32):
    append_case(spans, C, 4, 2, 64, f32, seed=C + len(spans))


def test_append_rows_in_any_order():
    append_case([(3, 71), (0, 40), (250, 33)], 16, 6, 2, 128, True, seed=5, shuffle=True)


def test_append_separate_rows_without_queries():
    append_case([(3, 71), (0, 40)], 32, 0, 4, 64, True, seed=6, fused=False)
    append_case([(3, 71), (0, 40)], 32, 4, 4, 64, False, seed=7, fused=False)


LOW, TOP = -(1 << 31), (1 << 31) - 1


@pytest.mark.parametrize("f32", [True, False])
def test_append_rows_and_chunks_that_write_nothing(f32):
    """Padding rows, positions outside the rotary table or the chunk table, chunks without a slot."""
    extra = [(-1, 3), (2, 3), (LOW, 0), (TOP, 0), (0, -1), (0, LOW), (1, TOP), (0, 400), (1, 303)]
    bad = [(0, 1, -1), (1, 0, LOW), (1, 18, TOP)]
    append_case([(10, 60), (0, 303)], 16, 4, 2, 64, f32, seed=8, shuffle=True, extra=extra, bad_slots=bad)
    append_case([(10, 60), (0, 303)], 16, 4, 2, 64, f32, seed=9, extra=extra, bad_slots=bad + [(0, 2, 41)])


def test_append_not_numbers_and_large_values():
    """Infinities and NaN go where the formula sends them; values beyond f16 become infinite."""
    nkv, hd, C = 1, 64, 16
    rng = np.random.default_rng(10)
    k, v = (rng.standard_normal((16, hd)).astype(np.float32) for _ in range(2))
    k[3, 5], k[4, 40], v[2, 7], v[9, 0], v[11, 1] = np.inf, np.nan, np.nan, -np.inf, 1e6
    slab, table = np.zeros((1, 2 * C * hd), np.float16), np.zeros((1, 1), np.int32)
    seq, pos, rope = np.zeros(16, np.int32), np.arange(16, dtype=np.int32), rope_table(16, hd)
    with np.errstate(over="ignore", invalid="ignore"):
        ref, bound, *_ = append_oracle(k, v, None, seq, pos, rope, slab, table, C, nkv, hd)
    got, _ = append_run(k, v, None, seq, pos, rope, slab, table, C, nkv, hd, True, False)
    close(got, ref, bound, "slab")


def test_append_offsets_past_32_bits():
    """A slab of more than 4 GiB: slots at its end."""
    torch = torch_cuda()
    nkv, hd, C = 8, 128, 256
    n_slots = 4200                                  # 1 MiB each
    slab = torch.zeros(n_slots, 2 * C * nkv * hd, device="cuda", dtype=torch.float16)
    rng = np.random.default_rng(11)
    pos = np.arange(250, 262, dtype=np.int32)
    k, v = (rng.standard_normal((12, nkv * hd)).astype(np.float32) for _ in range(2))
    rope, table = rope_table(300, hd), np.array([[n_slots - 1, n_slots - 2]], np.int32)
    dk, dv, ds, dp, dr, dt = dev(k), dev(v), dev(np.zeros(12, np.int32)), dev(pos), dev(rope), dev(table)
    mz.mz_kv_append(12, dk.data_ptr(), dv.data_ptr(), ds.data_ptr(), dp.data_ptr(), dr.data_ptr(), 300, slab.data_ptr(),
                    n_slots, dt.data_ptr(), 1, 2, C, nkv, hd, stream())
    torch.cuda.synchronize()
    small = np.zeros((2, 2 * C * nkv * hd), np.float16)
    ref, bound, *_ = append_oracle(k, v, None, np.zeros(12), pos, rope, small, np.array([[1, 0]]), C, nkv, hd)
    close(slab[-2:], ref, bound, "last slots")
    assert int(slab[:-2].count_nonzero()) == 0


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 17, 130, 1100])
def test_append_leaves_the_bits_of_the_projections_epilogues(m, hd):
    """Rows of a projection's fp32 output, appended, leave the slab and the queries that the rotary epilogues of the
    same products leave, bit for bit: chunks may be written by either."""
    torch = torch_cuda()
    K, C, dq, dkv, n_rope = 512, 16, 512, 256, 1500
    gen = torch.Generator(device="cuda").manual_seed(m + hd)
    x = torch.randn(m, K, device="cuda", generator=gen).half()

    def weights(n):
        w = torch.randint(0, 256, (n // 256, K // 64, 9216), device="cuda", dtype=torch.uint8, generator=gen)
        sc = (torch.rand(n // 256, K // 64, 512, device="cuda", generator=gen) * 0.01 + 0.01).half()
        w[..., 8192:] = sc.view(torch.uint8).view(n // 256, K // 64, 1024)
        return w

    wq, wkv, cs = weights(dq), weights(2 * dkv), dev(rope_table(n_rope, hd))
    pos = torch.arange(7, 7 + m, device="cuda", dtype=torch.int32)
    n_table = (7 + m + C - 1) // C
    table = torch.randperm(n_table + 3, device="cuda", generator=gen)[:n_table].int()
    slot_halves = 2 * C * dkv
    off = table[pos.long() // C].long() * slot_halves * 2 + (pos.long() % C) * dkv * 2
    slabs = [torch.full((n_table + 3, slot_halves), 7.0, device="cuda", dtype=torch.float16) for _ in range(2)]
    qs = [torch.zeros(m, dq, device="cuda", dtype=torch.float16) for _ in range(2)]
    rotary = dict(pos=pos.data_ptr(), rope_cs=cs.data_ptr(), head_dim=hd)
    mz.mz_q4_gemm_ex(x.data_ptr(), m, dq, K, wq.data_ptr(), 4, qs[0].data_ptr(), stream(), n_valid=dq, **rotary)
    mz.mz_q4_gemm_ex(x.data_ptr(), m, 2 * dkv, K, wkv.data_ptr(), 5, 0, stream(), n_valid=2 * dkv, kv_off=off.data_ptr(),
                     slab=slabs[0].data_ptr(), chunk_tokens=C, **rotary)
    q, kv = torch.zeros(m, dq, device="cuda"), torch.zeros(m, 2 * dkv, device="cuda")
    mz.mz_q4_gemm_ex(x.data_ptr(), m, dq, K, wq.data_ptr(), 0, q.data_ptr(), stream())
    mz.mz_q4_gemm_ex(x.data_ptr(), m, 2 * dkv, K, wkv.data_ptr(), 0, kv.data_ptr(), stream())
    seq = torch.zeros(m, device="cuda", dtype=torch.int32)
    mz.mz_kv_append(m, kv.data_ptr(), kv.data_ptr() + dkv * 4, seq.data_ptr(), pos.data_ptr(), cs.data_ptr(), n_rope,
                    slabs[1].data_ptr(), n_table + 3, table.data_ptr(), 1, n_table, C, dkv // hd, hd, stream(),
                    q_ptr=q.data_ptr(), n_q=dq // hd, q_out_ptr=qs[1].data_ptr(), k_stride=2 * dkv, v_stride=2 * dkv)
    torch.cuda.synchronize()
    for what, (a, b) in (("queries", qs), ("slab", slabs)):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)), what
    assert int((slabs[1] != 7).sum()) > m * 2 * dkv * 0.99


def test_append_captured_on_another_stream():
    """One graph serves every step: sequences, positions and rows change between its replays."""
    torch = torch_cuda()
    nq, nkv, hd, C, m, n_seq = 4, 2, 64, 16, 6, 6
    rng = np.random.default_rng(12)
    table = rng.permutation(n_seq * 8).reshape(n_seq, 8).astype(np.int32)
    rope, slab0 = rope_table(128, hd), np.zeros((n_seq * 8, 2 * C * nkv * hd), np.float16)
    slab, d_rope, d_table = dev(slab0), dev(rope), dev(table)
    rows = torch.zeros(m, (nq + 2 * nkv) * hd, device="cuda")
    seq, pos = torch.zeros(m, device="cuda", dtype=torch.int32), torch.zeros(m, device="cuda", dtype=torch.int32)
    q_out = torch.zeros(m, nq * hd, device="cuda", dtype=torch.float16)
    wide = rows.shape[1]

    def call():
        b = rows.data_ptr()
        mz.mz_kv_append(m, b + nq * hd * 4, b + (nq + nkv) * hd * 4, seq.data_ptr(), pos.data_ptr(), d_rope.data_ptr(), 128,
                        slab.data_ptr(), n_seq * 8, d_table.data_ptr(), n_seq, 8, C, nkv, hd, stream(), q_ptr=b, n_q=nq,
                        q_out_ptr=q_out.data_ptr(), k_stride=wide, v_stride=wide, q_stride=wide)

    call()
    torch.cuda.synchronize()
    slab.zero_()
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(g, stream=side):
        call()
    ref = slab0
    for step in range(4):
        x = rng.standard_normal((m, wide)).astype(np.float32)
        s, p = rng.permutation(n_seq).astype(np.int32), rng.integers(0, 128, m).astype(np.int32)
        rows.copy_(dev(x)), seq.copy_(dev(s)), pos.copy_(dev(p))
        before = slab.cpu().numpy()
        g.replay()
        torch.cuda.synchronize()
        q, k, v = np.split(x, [nq * hd, (nq + nkv) * hd], 1)
        ref, bound, qr, qb, _ = append_oracle(k, v, q, s, p, rope, before, table, C, nkv, hd)
        close(slab, ref, bound, f"slab of step {step}")
        close(q_out, qr, qb, f"q of step {step}")


# ----------------------------------------------------------------------------- attention

def attention_oracle(q, lens, slab, table, C, nq, nkv, hd):
    """(out, bound): weights rounded to f16 (u16 relative, the sums with them) from fp32 scores, f16 outputs."""
    n_seq, n_slots, dkv, group = len(lens), slab.shape[0], nkv * hd, nq // nkv
    out, bound = np.zeros((n_seq, nq * hd)), np.zeros((n_seq, nq * hd))
    halves = slab.reshape(n_slots, 2, C * dkv)
    ks, vs = halves[:, 0].reshape(n_slots, C, dkv), halves[:, 1].reshape(n_slots, dkv, C)
    for b in range(n_seq):
        n = min(max(int(lens[b]), 0), table.shape[1] * C)
        keep = [c for c in range((n + C - 1) // C) if 0 <= int(table[b, c]) < n_slots]
        at = np.concatenate([np.arange(c * C, min(n, (c + 1) * C)) for c in keep]) if keep else np.zeros(0, int)
        if at.size == 0:
            continue
        slots = table[b, at // C]
        k, v = ks[slots, at % C], vs[slots, :, at % C]
        k, v = k.astype(np.float64).reshape(-1, nkv, hd), v.astype(np.float64).reshape(-1, nkv, hd)
        for h in range(nq):
            x = q[b, h * hd:(h + 1) * hd].astype(np.float64)
            kk, vv = k[:, h // group], v[:, h // group]
            with np.errstate(invalid="ignore", over="ignore"):
                s = kk @ x / np.sqrt(hd)
                w = np.exp(s - s.max())
                p = w / w.sum()
                o = p @ vv
                # fp32 sums of hd exact products, the scale's and the exponent's roundings; a score of -inf is a
                # weight of exactly 0 on both sides, so its key adds no error (and no finite product to bound it by)
                on = np.isfinite(s)
                if on.any():
                    part = (np.abs(kk[on]) @ np.abs(x)).max() / np.sqrt(hd)
                    e = (hd + 4) * U32 * part + 4 * U32 * np.abs(s[on] - s[on].max()).max() + 4 * U32
                    bound[b, h * hd:(h + 1) * hd] = 2.1 * (U16 + e) * (p[on] @ np.abs(vv[on])) + U16 * np.abs(o) + TINY16 + \
                        len(s) * 2.0 ** -39 * np.abs(vv[on]).max(0)
                out[b, h * hd:(h + 1) * hd] = o
    return out, bound


def attention_run(q, lens, slab, table, C, nq, nkv, hd, ws=None):
    torch = torch_cuda()
    n_seq = len(lens)
    need = mz.mz_attention_batch_workspace_bytes(n_seq, nq, nkv, hd)
    if ws is None:
        ws = torch.full((need // 4 + 1,), float("nan"), device="cuda")      # what it held must not show
    out = torch.full((n_seq, nq * hd), 7.0, device="cuda", dtype=torch.float16)
    a = [dev(x) if isinstance(x, np.ndarray) else x for x in (q, lens, slab, table)]
    mz.mz_attention_batch(a[0].data_ptr(), a[1].data_ptr(), n_seq, a[2].data_ptr(), slab.shape[0], a[3].data_ptr(),
                          table.shape[1], C, nq, nkv, hd, ws.data_ptr(), need, out.data_ptr(), stream())
    torch.cuda.synchronize()
    return out


def attention_inputs(lens, C, nq, nkv, hd, seed, spread=1.0, extra_table=2):
    rng = np.random.default_rng(seed)
    lens = np.array(lens, np.int32)
    n_table = max(int(lens.max()), 1) // C + 1 + extra_table
    n_slots = int(sum((max(int(n), 0) + C - 1) // C for n in lens)) + 2
    order, at = rng.permutation(n_slots), 0
    table = rng.integers(-(1 << 31), 1 << 31, (len(lens), n_table)).astype(np.int32)   # entries past a length are never followed
    slab = np.full((n_slots, 2, C * nkv * hd), np.nan, np.float16)                     # nor what slots hold past it
    for b, n in enumerate(lens):
        for c in range((max(int(n), 0) + C - 1) // C):
            slot, held = order[at], min(C, n - c * C)
            at += 1
            table[b, c] = slot
            slab[slot, 0].reshape(C, -1)[:held] = rng.standard_normal((held, nkv * hd)) * spread
            slab[slot, 1].reshape(-1, C)[:, :held] = rng.standard_normal((nkv * hd, held))
    q = (rng.standard_normal((len(lens), nq * hd)) * spread).astype(np.float16)
    return q, lens, slab.reshape(n_slots, -1), table


def attention_case(lens, C, nq, nkv, hd, seed, spread=1.0):
    report("attention", lens=list(lens)[:12], n_seq=len(lens), C=C, nq=nq, nkv=nkv, hd=hd, seed=seed)
    a = attention_inputs(lens, C, nq, nkv, hd, seed, spread)
    out = attention_run(*a, C, nq, nkv, hd)
    ref, bound = attention_oracle(*a, C, nq, nkv, hd)
    close(out, ref, bound, "out")
    assert torch_cuda().equal(out, attention_run(*a, C, nq, nkv, hd)), "another run, other bits"
    return a, out


RAGGED = [0, 1, 2, 7, 8, 9, 31, 32, 33, 63, 127, 128, 129, 255, 300, 1000, 0, 5]


@pytest.mark.parametrize("nq,nkv,hd", [(4, 2, 64), (32, 8, 64), (12, 2, 128), (32, 8, 128), (16, 1, 128), (8, 8, 64),
                                       (3, 1, 64), (7, 1, 128), (33, 3, 64)])
@pytest.mark.parametrize("C", [8, 16, 32, 256])
def test_attention_ragged(nq, nkv, hd, C):
    attention_case(RAGGED, C, nq, nkv, hd, seed=nq * C + hd)


@pytest.mark.parametrize("lens,C,nq,nkv,hd", [
    ([1], 16, 4, 2, 64), ([5000], 64, 8, 2, 128), ([20000], 256, 6, 1, 128), ([3333, 1], 128, 2, 2, 64),
    ([0, 0, 9000, 0], 8, 5, 1, 64)])
def test_attention_few_long(lens, C, nq, nkv, hd):
    attention_case(lens, C, nq, nkv, hd, seed=sum(lens))


def test_attention_many_sequences():
    """More sequences than a workgroup has threads, some of them empty, more pairs than workgroups."""
    rng = np.random.default_rng(3)
    attention_case([int(n) for n in rng.integers(0, 200, 700)], 16, 4, 2, 64, seed=4)
    attention_case([0] * 600 + [77] + [0] * 300, 16, 4, 2, 64, seed=5)
    attention_case([0, 0, 0], 16, 4, 2, 64, seed=6)


def test_attention_sharp_and_flat():
    attention_case([700, 64, 3], 64, 8, 2, 128, seed=7, spread=4.0)
    attention_case([9000], 64, 4, 1, 64, seed=8, spread=0.01)


@pytest.mark.parametrize("n_seq", [63, 64, 65, 257, 700])
def test_attention_padded_batch(n_seq):
    """Few sequences with keys, far apart, first and last or in the middle: shares span runs of empty ones."""
    for at in ([0, n_seq - 1], [n_seq // 2], [1, 2, n_seq - 62, n_seq - 2] if n_seq > 64 else [5, 40]):
        lens = [0] * n_seq
        for i, b in enumerate(at):
            lens[b] = 130 + 97 * i
        attention_case(lens, 16, 4, 2, 64, seed=n_seq)


def test_attention_lengths_outside_the_table():
    a = list(attention_inputs([64, 40, 16], 16, 4, 2, 64, seed=9, extra_table=-1))
    assert a[3].shape[1] == 4
    a[1] = np.array([1 << 30, -5, 16], np.int32)
    out = attention_run(*a, 16, 4, 2, 64)
    ref, bound = attention_oracle(*a, 16, 4, 2, 64)
    close(out, ref, bound, "out")
    assert int(out[1].count_nonzero()) == 0


@pytest.mark.parametrize("C", [8, 16, 32, 64])
def test_attention_chunks_without_a_slot(C):
    """Their keys are left out; a sequence of none but such chunks gives zeros."""
    a = attention_inputs([500, 130, 100, 64], C, 4, 2, 64, seed=10)
    low, top = -(1 << 31), (1 << 31) - 1
    a[3][0, 0], a[3][0, 3], a[3][0, 500 // C] = -1, a[2].shape[0], low
    a[3][1, 1] = top
    a[3][2, :] = -1
    out = attention_run(*a, C, 4, 2, 64)
    ref, bound = attention_oracle(*a, C, 4, 2, 64)
    close(out, ref, bound, "out")
    assert int(out[2].count_nonzero()) == 0


@pytest.mark.parametrize("C", [16, 64])
def test_attention_not_numbers(C):
    """NaN, infinities and lowest values among the keys and values that count."""
    nq, nkv, hd = 4, 1, 64
    q, lens, slab, table = attention_inputs([90, 90, 90, 90, 90, 90, 90], C, nq, nkv, hd, seed=11)
    k = lambda b, j: slab[table[b, j // C], :C * hd].reshape(C, hd)[j % C]       # noqa: E731
    v = lambda b, j: slab[table[b, j // C], C * hd:].reshape(hd, C)[:, j % C]    # noqa: E731
    k(0, 50)[3] = np.nan
    v(1, 20)[5] = np.nan
    v(2, 33)[6] = np.inf
    v(2, 34)[6] = -np.inf
    v(2, 35)[7] = -np.inf
    k(3, 10)[:] = 65504.0                        # scores of either sign, far beyond the others
    k(4, 11)[:] = -65504.0
    q[5] = 1.0
    for j in range(90):                          # a row that sees nothing above -inf
        k(5, j)[0] = -np.inf
    q[6] = 1.0
    k(6, 77)[0] = -np.inf                        # one such key counts for nothing
    out = attention_run(q, lens, slab, table, C, nq, nkv, hd)
    ref, bound = attention_oracle(q, lens, slab, table, C, nq, nkv, hd)
    close(out, ref, bound, "out")


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("C", [8, 32, 256])
def test_attention_weights_keep_their_bits(C, hd):
    """Values that cancel: what weights lose shows beside an output near 0, as weights of 11 bits (2^-12 of each) would."""
    nq, nkv, lens = 8, 2, [2, 4, 10, 32, 64, 130, 300]
    q, lens, slab, table = attention_inputs(lens, C, nq, nkv, hd, seed=20)
    rng = np.random.default_rng(21)
    q = np.zeros_like(q).reshape(len(lens), nq, hd)      # a score is one product: q[0] k[0], q[0] at most 4
    q[:, :, 0] = rng.uniform(1, 4, q.shape[:2])
    ref, bound = np.zeros((len(lens), nq, hd)), np.zeros((len(lens), nq, hd))
    for b, n in enumerate(lens):
        k0 = (rng.uniform(0, 0.25, (n, nkv))).astype(np.float16)
        v = ((-1.0) ** np.arange(n)[:, None, None] * rng.uniform(1, 2, (1, nkv, hd))).astype(np.float16)
        for j in range(n):
            slot = slab[table[b, j // C]].reshape(2, -1)
            slot[0].reshape(C, nkv, hd)[j % C] = 0
            slot[0].reshape(C, nkv, hd)[j % C, :, 0] = k0[j]
            slot[1].reshape(nkv, hd, C)[:, :, j % C] = v[j]
        for h in range(nq):
            g = h // (nq // nkv)
            s = k0[:, g].astype(np.float64) * float(q[b, h, 0]) / np.sqrt(hd)
            w = np.exp(s - s.max())
            p = w / w.sum()
            size = p @ np.abs(v[:, g].astype(np.float64))
            ref[b, h] = p @ v[:, g].astype(np.float64)
            # exponents of at most 15 + 1.5 |s| <= 16: the scale, its product, the bias's sum and the difference are
            # rounded, 4 * 16 U32 in all, times ln 2; the exponential itself 2 U32; the weight's halves 2^-22; fp32
            # sums of n terms.  All that in numerator and denominator, then the output's own f16.
            e = 64 * 0.7 * U32 + 2 * U32 + 2.0 ** -22 + (n + 8) * U32
            bound[b, h] = 2.1 * e * size + U16 * np.abs(ref[b, h]) + TINY16
    out = attention_run(q.reshape(len(lens), -1), lens, slab, table, C, nq, nkv, hd)
    for b, n in enumerate(lens):
        close(out[b].view(nq, hd), ref[b], bound[b], f"{n} keys")


@pytest.mark.parametrize("C", [16, 64])
def test_attention_infinite_values(C):
    """Infinite values under weights that one f16 holds exactly (the largest is 1 beside itself) and under others."""
    nq, nkv, hd, n = 4, 1, 64, 70
    q, lens, slab, table = attention_inputs([1, n, n, n], C, nq, nkv, hd, seed=22)
    v = lambda b, j: slab[table[b, j // C], C * hd:].reshape(hd, C)[:, j % C]    # noqa: E731
    v(0, 0)[2], v(0, 0)[3] = np.inf, -np.inf
    q[1] = 0                                     # every weight the same
    v(1, 7)[4], v(1, 8)[5] = -np.inf, np.inf
    for j in range(n):
        v(2, j)[6] = np.inf
    v(3, 69)[7] = np.inf
    out = attention_run(q, lens, slab, table, C, nq, nkv, hd)
    close(out, *attention_oracle(q, lens, slab, table, C, nq, nkv, hd), "out")


def test_attention_against_the_single_sequence_call():
    torch = torch_cuda()
    nq, nkv, hd, C, n = 8, 2, 128, 64, 3000
    q, lens, slab, table = attention_inputs([n], C, nq, nkv, hd, seed=12)
    slab = np.nan_to_num(slab)
    out = attention_run(q, lens, slab, table, C, nq, nkv, hd)
    d = [dev(x) for x in (q, np.array([n - 1], np.int32), slab, table)]
    other = torch.zeros_like(out)
    mz.mz_attention(d[0].data_ptr(), d[1].data_ptr(), 1, d[2].data_ptr(), d[3].data_ptr(), (n + C - 1) // C, C, nq, nkv, hd,
                    other.data_ptr(), stream())
    torch.cuda.synchronize()
    ref, bound = attention_oracle(q, lens, slab, table, C, nq, nkv, hd)
    close(out, ref, bound, "batch")
    close(out, other.double().cpu().numpy(), 2 * bound, "batch against mz_attention")


def test_attention_offsets_past_32_bits():
    torch = torch_cuda()
    nq, nkv, hd, C, n = 8, 8, 128, 256, 700
    n_slots = 4200                                  # 1 MiB each
    slab = torch.zeros(n_slots, 2 * C * nkv * hd, device="cuda", dtype=torch.float16)
    q, lens, small, table = attention_inputs([n], C, nq, nkv, hd, seed=13)
    slab[n_slots - small.shape[0]:] = dev(small)
    far = table.copy()
    far[0, :3] += n_slots - small.shape[0]
    out = attention_run(q, lens, slab, far, C, nq, nkv, hd)
    ref, bound = attention_oracle(q, lens, small, table, C, nq, nkv, hd)
    close(out, ref, bound, "out")


def test_attention_as_many_queries_as_a_launch_holds():
    """2^24 - 16 query rows; three sequences have keys, the first and the last among them."""
    torch = torch_cuda()
    nq, nkv, hd, C, n_seq = 16, 1, 64, 16, (1 << 20) - 1
    q, lens, slab, table = attention_inputs([40, 1, 300], C, nq, nkv, hd, seed=17)
    at = [0, 70000, n_seq - 1]
    ref, bound = attention_oracle(q, lens, slab, table, C, nq, nkv, hd)
    all_q = torch.zeros(n_seq, nq, hd, device="cuda", dtype=torch.float16)
    all_lens = torch.zeros(n_seq, device="cuda", dtype=torch.int32)
    all_table = torch.full((n_seq, table.shape[1]), -1, device="cuda", dtype=torch.int32)
    all_q[at], all_lens[at], all_table[at] = dev(q).view(3, nq, hd), dev(lens), dev(table)
    need = mz.mz_attention_batch_workspace_bytes(n_seq, nq, nkv, hd)
    ws, d_slab = torch.empty(need, device="cuda", dtype=torch.uint8), dev(slab)
    out = torch.full((n_seq, nq * hd), 7.0, device="cuda", dtype=torch.float16)
    mz.mz_attention_batch(all_q.data_ptr(), all_lens.data_ptr(), n_seq, d_slab.data_ptr(), slab.shape[0], all_table.data_ptr(),
                          table.shape[1], C, nq, nkv, hd, ws.data_ptr(), need, out.data_ptr(), stream())
    torch.cuda.synchronize()
    close(out[at].view(ref.shape), ref, bound, "out")
    out[at] = 0
    assert not out.any()


def test_attention_captured_on_another_stream():
    """One graph over changing lengths; its workspace holds the last replay's partials."""
    torch = torch_cuda()
    nq, nkv, hd, C = 4, 2, 64, 16
    q, lens, slab, table = attention_inputs([800, 650, 513, 77], C, nq, nkv, hd, seed=14)
    need = mz.mz_attention_batch_workspace_bytes(4, nq, nkv, hd)
    ws = torch.full((need // 4,), float("nan"), device="cuda")
    d = [dev(x) for x in (q, lens, slab, table)]
    out = torch.zeros(4, nq * hd, device="cuda", dtype=torch.float16)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        mz.mz_attention_batch(d[0].data_ptr(), d[1].data_ptr(), 4, d[2].data_ptr(), slab.shape[0], d[3].data_ptr(),
                              table.shape[1], C, nq, nkv, hd, ws.data_ptr(), need, out.data_ptr(), stream())
    for now in ([800, 650, 513, 77], [1, 0, 300, 77], [0, 0, 0, 0], [128, 129, 1, 64]):
        now = np.array(now, np.int32)
        d[1].copy_(dev(now))
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        ref, bound = attention_oracle(q, now, slab, table, C, nq, nkv, hd)
        close(out, ref, bound, f"lengths {now.tolist()}")


def test_attention_on_two_streams_at_once():
    torch = torch_cuda()
    nq, nkv, hd, C = 8, 2, 128, 64
    sides = [torch.cuda.Stream() for _ in range(2)]
    args = [attention_inputs([4000 + 900 * i, 50, 3100], C, nq, nkv, hd, seed=15 + i) for i in range(2)]
    need = mz.mz_attention_batch_workspace_bytes(3, nq, nkv, hd)
    held = [[dev(x) for x in a] + [torch.full((need // 4,), float("nan"), device="cuda"),
                                   torch.zeros(3, nq * hd, device="cuda", dtype=torch.float16)] for a in args]
    torch.cuda.synchronize()
    for _ in range(5):
        for side, a, d in zip(sides, args, held):
            mz.mz_attention_batch(d[0].data_ptr(), d[1].data_ptr(), 3, d[2].data_ptr(), a[2].shape[0], d[3].data_ptr(),
                                  a[3].shape[1], C, nq, nkv, hd, d[4].data_ptr(), need, d[5].data_ptr(), side.cuda_stream)
    torch.cuda.synchronize()
    for i, (a, d) in enumerate(zip(args, held)):
        ref, bound = attention_oracle(*a, C, nq, nkv, hd)
        close(d[5], ref, bound, f"stream {i}")


# ----------------------------------------------------------------------------- adapters

def lora_oracle(x, adapter, a, b, scale, rank, base, n):
    """(y, bound): fp32 sums of k and of the ranks' products, nothing rounded to f16."""
    y, bound = base.astype(np.float64), np.zeros(base.shape)
    na, R, k = a.shape
    with np.errstate(invalid="ignore", over="ignore"):
        for i in range(na):
            rows, r = np.nonzero(adapter == i)[0], R if rank is None else min(max(int(rank[i]), 0), R)
            s = 1.0 if scale is None else float(scale[i])
            xs, ai, bi = x[rows].astype(np.float64), a[i, :r].astype(np.float64), b[i, :, :r].astype(np.float64)
            y[rows, :n] += s * ((xs @ ai.T) @ bi.T)
            size = abs(s) * ((np.abs(xs) @ np.abs(ai).T) @ np.abs(bi).T)
            bound[rows, :n] = 2 * (k + R + 20) * U32 * size + 2 * U32 * np.abs(y[rows, :n])
    return y, bound


def lora_run(x, adapter, a, b, scale, rank, base, n, in_place=False, ws=None):
    torch = torch_cuda()
    m, k = x.shape
    na, R, _ = a.shape
    need = mz.mz_lora_workspace_bytes(m, k, R, na)
    if ws is None:
        ws = torch.full((need // 4,), float("nan"), device="cuda")
    d = [None if v is None else dev(v) for v in (x, adapter, a, b, scale, rank, base)]
    y = d[6] if in_place else torch.full(base.shape, 7.0, device="cuda")
    mz.mz_lora_add(d[0].data_ptr(), m, k, d[1].data_ptr(), na, d[2].data_ptr(), d[3].data_ptr(), R, n, d[6].data_ptr(),
                   y.data_ptr(), base.shape[1], ws.data_ptr(), need, stream(),
                   scale_ptr=0 if scale is None else d[4].data_ptr(), rank_ptr=0 if rank is None else d[5].data_ptr())
    torch.cuda.synchronize()
    return y


def lora_inputs(adapter, k, n, R, na, seed, stride=None, ranks=None):
    rng = np.random.default_rng(seed)
    adapter = np.array(adapter, np.int32)
    m = len(adapter)
    x = rng.standard_normal((m, k)).astype(np.float16)
    a = (rng.standard_normal((na, R, k)) / np.sqrt(k)).astype(np.float16)
    b = (rng.standard_normal((na, n, R)) * 0.3).astype(np.float16)
    scale = (rng.random(na) + 0.5).astype(np.float32)
    rank = np.array([int(rng.integers(0, R + 1)) for _ in range(na)] if ranks is None else ranks, np.int32)
    for i in range(na):                  # what lies past a rank is not data
        a[i, rank[i]:], b[i, :, rank[i]:] = np.nan, np.inf
    base = rng.standard_normal((m, stride or (n + 3) // 4 * 4)).astype(np.float32)
    return x, adapter, a, b, scale, rank, base, n


def lora_case(adapter, k, n, R, na, seed, **kw):
    torch = torch_cuda()
    a = lora_inputs(adapter, k, n, R, na, seed, **kw)
    report("lora", m=len(adapter), k=k, n=n, R=R, adapters=na, ranks=a[5].tolist()[:8], seed=seed)
    ref, bound = lora_oracle(*a)
    y = lora_run(*a)
    close(y[:, :n], ref[:, :n], bound[:, :n], "y")
    assert bool((y[:, n:] == 7).all()), "columns past n"
    bits = lambda t: t[:, :n].contiguous().view(torch.int32)  # noqa: E731
    assert torch.equal(bits(lora_run(*a)), bits(y)), "another run, other bits"
    there = lora_run(*a, in_place=True)
    assert torch.equal(bits(there), bits(y)), "in place"
    assert torch.equal(there[:, n:], dev(a[6])[:, n:]), "columns past n in place"
    none = dev((a[1] < 0) | (a[1] >= na))
    assert torch.equal(bits(y)[none], bits(dev(a[6]))[none]), "rows without an adapter"


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 33, 64, 65, 200])
@pytest.mark.parametrize("k,n,R", [(64, 256, 16), (264, 100, 8), (2048, 515, 32)])
def test_lora_mixed_rows(m, k, n, R):
    rng = np.random.default_rng(m)
    lora_case(rng.integers(-1, 6, m), k, n, R, 5, seed=m + k)      # -1 and 5: none


@pytest.mark.parametrize("R", [8, 16, 24, 32, 40, 64, 72, 128])
def test_lora_ranks(R):
    rng = np.random.default_rng(R)
    ranks = [0, 1, R // 2, R - 1, R, min(R, 15), min(R, 17)]
    lora_case(rng.integers(-1, 7, 40), 136, 77, R, 7, seed=R, ranks=ranks)
    lora_case(rng.integers(0, 7, 600), 136, 77, R, 7, seed=R + 1, ranks=ranks)


def test_lora_one_adapter_for_all():
    lora_case([0] * 1, 8, 1, 8, 1, seed=20)
    lora_case([0] * 47, 512, 256, 16, 1, seed=21)
    lora_case([1] * 512, 512, 256, 16, 2, seed=22)
    lora_case([1] * 1100, 512, 256, 16, 2, seed=23)


def test_lora_no_adapters_used():
    lora_case([-1] * 5, 64, 60, 16, 2, seed=24)
    lora_case([-1] * 700, 64, 60, 16, 2, seed=25)
    lora_case([-1] * 130 + [1] + [2] * 70, 64, 60, 16, 2, seed=25)
    lora_case([7] * 5 + [-(1 << 31), (1 << 31) - 1], 64, 60, 16, 2, seed=26)


@pytest.mark.parametrize("m", [64, 65, 129, 511, 512, 513, 576, 1025, 2000, 8192, 8193, 8300, 16500])
def test_lora_runs_of_rows(m):
    """Requests one after the other: a tile may hold the end of one and the beginning of the next."""
    rng = np.random.default_rng(m)
    cuts = np.sort(rng.integers(0, m, 6))
    lora_case(np.searchsorted(cuts, np.arange(m), side="right") - 1, 320, 300, 32, 7, seed=m, stride=512)
    lora_case(rng.integers(-1, 4, m), 320, 300, 16, 4, seed=m + 1)


@pytest.mark.parametrize("m", [65, 300, 1000])
def test_lora_many_adapters(m):
    """More adapters than rows, one for each row, and the most a call takes."""
    rng = np.random.default_rng(m)
    lora_case(rng.permutation(2 * m)[:m], 40, 20, 8, 2 * m, seed=m)
    lora_case(rng.integers(-3, 2050, m), 16, 12, 8, 2047, seed=m + 1)


@pytest.mark.parametrize("m,n,R", [(1024, 4100, 64), (1030, 4097, 104), (2100, 2048, 128)])
def test_lora_many_rows_and_columns(m, n, R):
    """Wide ranges of the second product, the last of them short."""
    rng = np.random.default_rng(m)
    lora_case(rng.integers(-1, 3, m), 40, n, R, 3, seed=m, stride=(n + 7) // 4 * 4)
    lora_case(np.arange(m) * 4 // m - 1, 24, n, R, 3, seed=m + 1)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_lora_list_off_16_bytes(shift):
    torch = torch_cuda()
    rng = np.random.default_rng(34)
    for m in (66, 1027):
        x, adapter, a, b, scale, rank, base, n = lora_inputs(rng.integers(-1, 3, m), 64, 32, 16, 3, seed=35)
        need = mz.mz_lora_workspace_bytes(m, 64, 16, 3)
        ws = torch.full((need // 4,), float("nan"), device="cuda")
        ids = torch.full((shift + m,), 1, device="cuda", dtype=torch.int32)
        ids[shift:] = dev(adapter)
        d = [dev(v) for v in (x, a, b, scale, rank, base)]
        y = torch.zeros(base.shape, device="cuda")
        mz.mz_lora_add(d[0].data_ptr(), m, 64, ids[shift:].data_ptr(), 3, d[1].data_ptr(), d[2].data_ptr(), 16, n, d[5].data_ptr(),
                       y.data_ptr(), base.shape[1], ws.data_ptr(), need, stream(), scale_ptr=d[3].data_ptr(),
                       rank_ptr=d[4].data_ptr())
        torch.cuda.synchronize()
        close(y, *lora_oracle(x, adapter, a, b, scale, rank, base, n), f"{m} rows")


def test_lora_many_rows_replayed_over_other_lists():
    """One graph of 500 rows: lists in runs, mixed, of one adapter and of none."""
    torch = torch_cuda()
    rng = np.random.default_rng(36)
    m, k, na = 500, 128, 5
    x, adapter, a, b, scale, rank, base, n = lora_inputs([0] * m, k, 300, 64, na, seed=36, ranks=[64, 9, 0, 33, 48])
    need = mz.mz_lora_workspace_bytes(m, k, 64, na)
    ws = torch.full((need // 4,), float("nan"), device="cuda")
    d = [dev(v) for v in (x, adapter, a, b, scale, rank, base)]
    y = torch.zeros(base.shape, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        mz.mz_lora_add(d[0].data_ptr(), m, k, d[1].data_ptr(), na, d[2].data_ptr(), d[3].data_ptr(), 64, n, d[6].data_ptr(),
                       y.data_ptr(), base.shape[1], ws.data_ptr(), need, stream(), scale_ptr=d[4].data_ptr(),
                       rank_ptr=d[5].data_ptr())
    for ids in (np.arange(m) * na // m, rng.integers(-1, na, m), np.full(m, 3), np.full(m, -1), np.arange(m) // 7 % na):
        ids = ids.astype(np.int32)
        d[1].copy_(dev(ids))
        y.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        ref, bound = lora_oracle(x, ids, a, b, scale, rank, base, n)
        close(y[:, :n], ref[:, :n], bound[:, :n], "y")


def test_lora_without_scales_and_ranks():
    x, adapter, a, b, scale, rank, base, n = lora_inputs([1, 0, -1, 1, 1], 96, 48, 16, 2, seed=27, ranks=[16, 16])
    ref, bound = lora_oracle(x, adapter, a, b, None, None, base, n)
    close(lora_run(x, adapter, a, b, None, None, base, n), ref, bound, "y")


@pytest.mark.parametrize("m", [40, 700])
def test_lora_rows_do_not_touch_each_other(m):
    """Rows of NaN, infinities and large values among others, and an adapter that holds them."""
    rng = np.random.default_rng(28)
    x, adapter, a, b, scale, rank, base, n = lora_inputs(rng.integers(0, 4, m), 256, 128, 16, 4, seed=28, ranks=[16] * 4)
    a[3, 2, 5], b[3, 7, 1] = np.inf, np.nan
    adapter[:9] = [0, 0, 1, 1, 2, -1, 2, 0, 3]
    x[1], x[3, 4], x[5], x[6, 1] = np.nan, np.inf, np.nan, 65504.0
    base[7, 3] = np.inf
    ref, bound = lora_oracle(x, adapter, a, b, scale, rank, base, n)
    close(lora_run(x, adapter, a, b, scale, rank, base, n), ref, bound, "y")


def test_lora_large_and_small_values():
    """x A^T far beyond f16 and below its normal range keeps fp32 precision."""
    x, adapter, a, b, scale, rank, base, n = lora_inputs([0, 1, 0, 1], 512, 64, 16, 2, seed=29, ranks=[16, 16])
    x[0], x[2] = np.float16(3000) * x[0], np.float16(2.0 ** -12) * x[2]
    a[0] = a[0] * np.float16(200)
    base[2] = 0
    scale[1] = -1e-20
    base[1] = 0
    ref, bound = lora_oracle(x, adapter, a, b, scale, rank, base, n)
    close(lora_run(x, adapter, a, b, scale, rank, base, n), ref, bound, "y")


@pytest.mark.parametrize("m,k,n,R", [(1, 64, 256, 16), (20, 64, 100, 32), (20, 4096, 130, 32), (64, 2048, 300, 128),
                                     (200, 64, 300, 16), (500, 328, 300, 40), (600, 64, 8200, 64), (530, 64, 8300, 128)])
def test_lora_small_ranks_meet_large_columns(m, k, n, R):
    """Ranks of t far below others of their row, with columns of B that make up for it.  In every third column the
    smallest rank, 2^-35 of the largest, counts alone, so that it needs bits of its own.  Fused, few-row and tile
    forms."""
    rng = np.random.default_rng(m + R)
    x, adapter, a, b, scale, rank, base, n = lora_inputs(rng.integers(-1, 3, m), k, n, R, 3, seed=37, ranks=[R, R - 3, 7])
    down = rng.integers(0, 20, (3, R))                       # t of rank r falls by 2^down, B rises by as much
    down[:, :2] = [[0, 22]] * 3
    a = (a.astype(np.float64) * 2.0 ** np.minimum(8 - down, 8)[:, :, None]).astype(np.float16)
    x[:, :k // 2] *= np.float16(2.0 ** 5)
    a[:, 1, :k // 2] = 0                                     # one rank that sees the small half of x only
    x[:, k // 2:] *= np.float16(2.0 ** -8)
    b = (b.astype(np.float64) * 2.0 ** (down - 12)[:, None, :]).astype(np.float16)
    for i, r in enumerate(rank):
        a[i, r:], b[i, :, r:] = np.nan, np.inf
        b[i, ::3, [j for j in range(R) if j != 1]] = 0
        b[i, 1::3, 0] = 2.0 ** -24
    base[: m // 2] = 0
    ref, bound = lora_oracle(x, adapter, a, b, scale, rank, base, n)
    y = lora_run(x, adapter, a, b, scale, rank, base, n)
    close(y[:, :n], ref[:, :n], bound[:, :n], "y")


@pytest.mark.parametrize("m", [3, 40, 130])
def test_lora_infinite_adapters(m):
    """Infinite values in B, in A and in x beside ranks that one part of them holds exactly."""
    x, adapter, a, b, scale, rank, base, n = lora_inputs([r % 2 for r in range(m)], 64, 48, 16, 2, seed=38, ranks=[16, 16])
    b[0, 5, 3], b[0, 6, 4], b[1, 7, 2] = np.inf, -np.inf, np.inf
    b[1, 8, :] = 0
    b[1, 9, 2] = 1
    a[:] = 0
    a[:, :, 0] = 1                              # t = x[0] for every rank: 1, a power of two, in the first rows
    x[:2, 0] = 1
    x[2, 0] = np.inf
    ref, bound = lora_oracle(x, adapter, a, b, scale, rank, base, n)
    close(lora_run(x, adapter, a, b, scale, rank, base, n), ref, bound, "y")


@pytest.mark.parametrize("m", [2, 40, 130])
def test_lora_scales_of_any_size(m):
    """Scales near the ends of fp32's range with B, or x, that brings the result back."""
    x, adapter, a, b, scale, rank, base, n = lora_inputs([r % 2 for r in range(m)], 64, 48, 16, 2, seed=39, ranks=[16, 11])
    scale[:] = [2.0 ** 122, 2.0 ** -120]
    x, base[:] = np.where(adapter[:, None] == 0, x * np.float16(2.0 ** 3), x * np.float16(2.0 ** 8)).astype(np.float16), 0
    b[0, :, :16] = (b[0, :, :16].astype(np.float64) * 2.0 ** -12).astype(np.float16)
    ref, bound = lora_oracle(x, adapter, a, b, scale, rank, base, n)
    close(lora_run(x, adapter, a, b, scale, rank, base, n), ref, bound, "y")


def test_lora_captured_on_another_stream():
    torch = torch_cuda()
    rng = np.random.default_rng(30)
    x, adapter, a, b, scale, rank, base, n = lora_inputs([0] * 30, 256, 200, 16, 3, seed=30, ranks=[16, 9, 4])
    need = mz.mz_lora_workspace_bytes(30, 256, 16, 3)
    ws = torch.full((need // 4,), float("nan"), device="cuda")
    d = [dev(v) for v in (x, adapter, a, b, scale, rank, base)]
    y = torch.zeros(base.shape, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        mz.mz_lora_add(d[0].data_ptr(), 30, 256, d[1].data_ptr(), 3, d[2].data_ptr(), d[3].data_ptr(), 16, n,
                       d[6].data_ptr(), y.data_ptr(), base.shape[1], ws.data_ptr(), need, stream(),
                       scale_ptr=d[4].data_ptr(), rank_ptr=d[5].data_ptr())
    for step in range(4):
        adapter = rng.integers(-1, 4, 30).astype(np.int32)
        x = rng.standard_normal(x.shape).astype(np.float16)
        d[0].copy_(dev(x)), d[1].copy_(dev(adapter))
        g.replay()
        torch.cuda.synchronize()
        ref, bound = lora_oracle(x, adapter, a, b, scale, rank, base, n)
        close(y, ref, bound, f"step {step}")


def test_lora_offsets_past_32_bits():
    """Adapters and rows beyond 4 GiB from their bases."""
    torch = torch_cuda()
    k, n, R, na = 16384, 64, 128, 1200
    a = torch.zeros(na, R, k, device="cuda", dtype=torch.float16)       # 4 MiB each
    b = torch.zeros(na, n, R, device="cuda", dtype=torch.float16)
    x, adapter, a1, b1, scale, rank, base, _ = lora_inputs([0, 0, -1], k, n, R, 1, seed=31, ranks=[R])
    a[-1], b[-1] = dev(a1[0]), dev(b1[0])
    need = mz.mz_lora_workspace_bytes(3, k, R, na)
    ws, y = torch.full((need // 4,), float("nan"), device="cuda"), torch.zeros(base.shape, device="cuda")
    d = [dev(v) for v in (x, np.where(adapter < 0, -1, na - 1).astype(np.int32), base)]
    mz.mz_lora_add(d[0].data_ptr(), 3, k, d[1].data_ptr(), na, a.data_ptr(), b.data_ptr(), R, n, d[2].data_ptr(),
                   y.data_ptr(), base.shape[1], ws.data_ptr(), need, stream())
    torch.cuda.synchronize()
    ref, bound = lora_oracle(x, adapter, a1, b1, None, None, base, n)
    close(y, ref, bound, "y")


@pytest.mark.parametrize("m,in_place", [(3, True), (3, False), (64, True), (70, True), (70, False), (600, True)])
def test_lora_rows_past_32_bits(m, in_place):
    """Rows of base and y whose last ones lie beyond 2^32 bytes, and beyond 2^31 elements, from the first."""
    torch = torch_cuda()
    k, n, R, na = 64, 300, 16, 4
    rng = np.random.default_rng(m)
    x, adapter, a, b, scale, rank, base, n = lora_inputs(rng.integers(-1, 4, m), k, n, R, na, seed=40)
    stride = ((1 << 31) // (m - 1) + 5) // 4 * 4 + 4
    assert (m - 1) * stride > 1 << 31
    far = torch.empty((m - 1) * stride + n, device="cuda")
    rows = far.as_strided((m, n), (stride, 1))
    rows.copy_(dev(base)[:, :n])
    out = far if in_place else torch.empty_like(far)
    need = mz.mz_lora_workspace_bytes(m, k, R, na)
    ws = torch.full((need // 4,), float("nan"), device="cuda")
    d = [dev(v) for v in (x, adapter, a, b, scale, rank)]
    mz.mz_lora_add(d[0].data_ptr(), m, k, d[1].data_ptr(), na, d[2].data_ptr(), d[3].data_ptr(), R, n, far.data_ptr(),
                   out.data_ptr(), stride, ws.data_ptr(), need, stream(), scale_ptr=d[4].data_ptr(), rank_ptr=d[5].data_ptr())
    torch.cuda.synchronize()
    ref, bound = lora_oracle(x, adapter, a, b, scale, rank, base, n)
    close(out.as_strided((m, n), (stride, 1)), ref[:, :n], bound[:, :n], "y")


@pytest.mark.parametrize("m", [3, 130])
def test_lora_adapters_past_32_bits(m):
    """A and B of the last adapter beyond 2^32 bytes from the first one's, in the forms of few and of many rows."""
    torch = torch_cuda()
    k, n, R, na = 16384, 16384, 128, 1100
    a = torch.zeros(na, R, k, device="cuda", dtype=torch.float16)       # 4 MiB each, as each of b
    b = torch.zeros(na, n, R, device="cuda", dtype=torch.float16)
    x, adapter, a1, b1, scale, rank, base, _ = lora_inputs([r % 3 - 1 for r in range(m)], k, n, R, 2, seed=41, ranks=[R, R])
    a[na - 2:], b[na - 2:] = dev(a1), dev(b1)
    need = mz.mz_lora_workspace_bytes(m, k, R, na)
    ws, y = torch.full((need // 4,), float("nan"), device="cuda"), torch.zeros(base.shape, device="cuda")
    d = [dev(v) for v in (x, np.where(adapter < 0, -1, na - 2 + adapter).astype(np.int32), base)]
    mz.mz_lora_add(d[0].data_ptr(), m, k, d[1].data_ptr(), na, a.data_ptr(), b.data_ptr(), R, n, d[2].data_ptr(),
                   y.data_ptr(), base.shape[1], ws.data_ptr(), need, stream())
    torch.cuda.synchronize()
    ref, bound = lora_oracle(x, adapter, a1, b1, None, None, base, n)
    close(y, ref, bound, "y")


def test_lora_rows_of_the_second_piece_past_32_bits():
    """More rows than one pass takes, x beyond 2^32 bytes."""
    torch = torch_cuda()
    m, k, n, R, na = 8192 + 70, 1 << 18, 12, 8, 2
    gen = torch.Generator(device="cuda").manual_seed(42)
    x = torch.randn(m, k, device="cuda", dtype=torch.float16, generator=gen)      # 4 GiB and more
    a = (torch.randn(na, R, k, device="cuda", generator=gen) / 512).half()
    b = torch.randn(na, n, R, device="cuda", generator=gen).half()
    adapter = torch.randint(-1, na, (m,), device="cuda", generator=gen).int()
    base = torch.randn(m, n, device="cuda", generator=gen)
    need = mz.mz_lora_workspace_bytes(m, k, R, na)
    ws, y = torch.full((need // 4,), float("nan"), device="cuda"), torch.zeros(m, n, device="cuda")
    mz.mz_lora_add(x.data_ptr(), m, k, adapter.data_ptr(), na, a.data_ptr(), b.data_ptr(), R, n, base.data_ptr(), y.data_ptr(),
                   n, ws.data_ptr(), need, stream())
    torch.cuda.synchronize()
    at = np.concatenate([np.arange(0, 70), np.arange(8100, m)])       # of both pieces, the last rows among them
    some = lambda t: t[dev(at)].cpu().numpy()                         # noqa: E731
    ref, bound = lora_oracle(some(x), some(adapter), a.cpu().numpy(), b.cpu().numpy(), None, None, some(base), n)
    close(some(y), ref, bound, "y")


@pytest.mark.parametrize("m,k,R", [(65, 14336, 16), (130, 8200, 32), (130, 14336, 64), (700, 8192, 24), (130, 2816, 16),
                                   (1300, 14336, 16)])
def test_lora_many_rows_in_many_splits(m, k, R):
    """K splits of the tiles' first product up to 32, odd counts and counts that do not divide the steps among them."""
    rng = np.random.default_rng(m + k)
    lora_case(rng.integers(-1, 3, m), k, 70, R, 3, seed=43)
    lora_case(np.arange(m) * 4 // m - 1, k, 70, R, 3, seed=44)


def test_lora_on_two_streams_at_once_and_a_larger_workspace():
    """Many rows, sorted tiles; the first call's workspace is one for 8192 rows."""
    torch = torch_cuda()
    k, n, R, na, streams, calls = 512, 600, 24, 5, [torch.cuda.Stream() for _ in range(2)], []
    for i, m in enumerate((700, 333)):
        x, adapter, a, b, scale, rank, base, _ = lora_inputs([(3 * r + i) % na for r in range(m)], k, n, R, na, seed=33 + i)
        need = mz.mz_lora_workspace_bytes(8192 if i == 0 else m, k, R, na)
        calls.append(([dev(v) for v in (x, adapter, a, b, scale, rank, base)], m, need,
                      torch.full((need // 4,), float("nan"), device="cuda"), torch.zeros(base.shape, device="cuda"),
                      lora_oracle(x, adapter, a, b, scale, rank, base, n)))
    torch.cuda.synchronize()
    for _ in range(20):
        for st, (d, m, need, ws, y, _) in zip(streams, calls):
            mz.mz_lora_add(d[0].data_ptr(), m, k, d[1].data_ptr(), na, d[2].data_ptr(), d[3].data_ptr(), R, n, d[6].data_ptr(),
                           y.data_ptr(), y.shape[1], ws.data_ptr(), need, st.cuda_stream, scale_ptr=d[4].data_ptr(),
                           rank_ptr=d[5].data_ptr())
    torch.cuda.synchronize()
    for _, _, _, _, y, (ref, bound) in calls:
        close(y, ref, bound, "y")


# ----------------------------------------------------------------------------- rules on logits

def logits_oracle(x, penalty, histories, biases, mask, mask_row):
    """(out, bound): at most five fp32 roundings of values no larger than the parts."""
    m, v = x.shape
    out, bound = x.astype(np.float64), np.zeros(x.shape)
    with np.errstate(all="ignore"):
        for i in range(m):
            rep, freq, pres = (float(t) for t in penalty[i])
            h = np.array([t for t in histories[i] if 0 <= t < v], np.int64)
            ids, c = np.unique(h, return_counts=True)
            old = out[i, ids]
            held = np.where(old > 0, old / rep, old * rep)
            out[i, ids] = held - freq * c - pres
            bound[i, ids] = 5 * U32 * (np.abs(held) + np.abs(freq * c) + abs(pres))
            last = {t: b for t, b in biases[i] if 0 <= t < v}
            for t, b in last.items():
                out[i, t] += b
                bound[i, t] += U32 * (abs(out[i, t]) + abs(b))
            if mask is not None and 0 <= mask_row[i] < len(mask):
                bits = np.unpackbits(mask[mask_row[i]].view(np.uint8), bitorder="little")[:v]
                out[i, bits == 0] = -np.inf
    return out, bound


def rows_of(lists, dtype):
    off = np.concatenate([[0], np.cumsum([len(t) for t in lists])]).astype(np.int64)
    flat = np.array([t for one in lists for t in one] + [0], dtype)      # never an empty buffer
    return flat, off


def logits_run(x, penalty, histories, biases, mask, mask_row, stride=None, mode="new", shift=0):
    """mode: "new" rows, "in place", or "token" only.  shift: floats before the first row (alignment)."""
    torch = torch_cuda()
    m, v = x.shape
    stride = stride or v
    rows = np.full((m, stride), 9.0, np.float32)
    rows[:, :v] = x
    buf = torch.full((shift + m * stride,), 5.0, device="cuda")
    buf[shift:] = dev(rows).view(-1)
    src = buf[shift:].view(m, stride)
    dst = torch.full((shift + m * stride,), 7.0, device="cuda")[shift:].view(m, stride) if mode == "new" else src
    need = mz.mz_logits_rules_workspace_bytes(m, v)
    ws, token = torch.full((need // 4,), float("nan"), device="cuda"), torch.full((m,), -7, device="cuda", dtype=torch.int32)
    kw, keep = {}, []
    if histories is not None:
        flat, off = rows_of(histories, np.int32)
        keep += [dev(flat), dev(off), dev(np.asarray(penalty, np.float32))]
        kw.update(history_ptr=keep[-3].data_ptr(), history_off_ptr=keep[-2].data_ptr(), penalty_ptr=keep[-1].data_ptr())
    if biases is not None:
        tok, off = rows_of([[t for t, _ in b] for b in biases], np.int32)
        val, _ = rows_of([[u for _, u in b] for b in biases], np.float32)
        keep += [dev(tok), dev(val), dev(off)]
        kw.update(bias_token_ptr=keep[-3].data_ptr(), bias_value_ptr=keep[-2].data_ptr(), bias_off_ptr=keep[-1].data_ptr())
    if mask is not None:
        keep += [dev(mask.view(np.int32)), dev(np.asarray(mask_row, np.int32))]
        kw.update(mask_ptr=keep[-2].data_ptr(), n_masks=mask.shape[0], mask_words=mask.shape[1], mask_row_ptr=keep[-1].data_ptr())
    mz.mz_logits_rules(src.data_ptr(), m, v, stride, None if mode == "token" else dst.data_ptr(), token.data_ptr(),
                       ws.data_ptr(), need, stream(), **kw)
    torch.cuda.synchronize()
    if mode == "token":
        assert torch.equal(src.contiguous().view(torch.int32), dev(rows.view(np.int32))), "the logits are only read"
    else:
        assert bool((dst[:, v:] == (7.0 if mode == "new" else 9.0)).all()), "columns past vocab"
    return dst[:, :v].cpu().numpy(), token.cpu().numpy()


def picked(out):
    """The lowest token of the largest value, NaN aside; -1 where nothing is above -inf."""
    best = np.where(np.isnan(out), -np.inf, out)
    return np.where(best.max(1) > -np.inf, best.argmax(1), -1)


def logits_inputs(m, v, seed, n_hist=50, n_bias=9, n_masks=3, low=0):
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((m, v)) * 3).astype(np.float32)
    penalty = np.stack([1 + rng.random(m), rng.random(m), rng.random(m) - 0.3], 1).astype(np.float32)
    # repeats, tokens outside the vocabulary, some empty lists
    histories = [[int(t) for t in (rng.random(int(rng.integers(0, n_hist + 1))) ** 3 * (v + 3) - low)] for _ in range(m)]
    biases = [[(int(rng.integers(-2, v + 2)), float(np.float32(rng.standard_normal()))) for _ in range(int(rng.integers(0, n_bias + 1)))]
              for _ in range(m)]
    mask = rng.integers(0, 1 << 32, (n_masks, (v + 31) // 32 + 1), dtype=np.uint32)
    mask_row = rng.integers(-1, n_masks + 1, m).astype(np.int32)
    return x, penalty, histories, biases, mask, mask_row


def logits_case(a, **kw):
    report("logits", m=a[0].shape[0], vocab=a[0].shape[1], kw=kw)
    none = [[] for _ in a[2] or a[0]]
    ref, bound = logits_oracle(a[0], a[1], a[2] or none, a[3] or none, a[4], a[5])
    out, token = logits_run(*a, **kw)
    close(out, ref, bound, "logits")
    assert np.array_equal(token, picked(out))
    assert np.array_equal(logits_run(*a, **{**kw, "mode": "in place"})[0].view(np.int32), out.view(np.int32)), "in place"
    assert np.array_equal(logits_run(*a, **{**kw, "mode": "token"})[1], token), "token only"
    return out, token


@pytest.mark.parametrize("m,v", [(1, 1), (1, 3), (2, 31), (3, 33), (1, 1000), (4, 1024), (2, 1025), (5, 4096), (3, 10007),
                                 (1, 128256), (200, 12345)])
def test_logits_rules(m, v):
    logits_case(logits_inputs(m, v, seed=m + v, low=2))


@pytest.mark.parametrize("v,stride,shift", [(1000, 1024, 0), (1001, 1024, 0), (1000, 1003, 0), (1000, 1024, 1), (4099, 4352, 4)])
def test_logits_strides_and_alignment(v, stride, shift):
    logits_case(logits_inputs(3, v, seed=v + stride), stride=stride, shift=shift)


@pytest.mark.parametrize("use", range(8))
def test_logits_rules_one_by_one(use):
    x, penalty, histories, biases, mask, mask_row = logits_inputs(6, 3000, seed=30)
    logits_case((x, penalty, histories if use & 1 else None, biases if use & 2 else None, mask if use & 4 else None,
                 mask_row if use & 4 else None))


def test_logits_long_histories():
    rng = np.random.default_rng(31)
    x, penalty, _, biases, mask, mask_row = logits_inputs(3, 5000, seed=31, n_bias=3000)
    histories = [[7] * 70000, [int(t) for t in rng.integers(0, 5000, 40000)], []]
    logits_case((x, penalty, histories, biases, mask, mask_row))


def test_logits_many_rows():
    """The larger slices, and rows enough for many workgroups."""
    logits_case(logits_inputs(130, 20000, seed=32, n_hist=300))


def test_logits_as_many_rows_as_a_launch_holds():
    torch = torch_cuda()
    m, v = (1 << 23) - 1, 5
    x = torch.randint(-4, 5, (m, v), device="cuda", dtype=torch.int32).float()
    need = mz.mz_logits_rules_workspace_bytes(m, v)
    ws, token = torch.empty(need, device="cuda", dtype=torch.uint8), torch.full((m,), -7, device="cuda", dtype=torch.int32)
    mask = dev(np.array([[0b11111], [0b01010], [0]], np.uint32).view(np.int32))
    mask_row = torch.arange(m, device="cuda", dtype=torch.int32) % 4          # 3: none
    mz.mz_logits_rules(x.data_ptr(), m, v, v, 0, token.data_ptr(), ws.data_ptr(), need, mask_ptr=mask.data_ptr(), n_masks=3,
                       mask_words=1, mask_row_ptr=mask_row.data_ptr(), stream=stream())
    torch.cuda.synchronize()
    weight = x * 8 - torch.arange(v, device="cuda")              # of equal values the lowest index
    want = weight.argmax(1)
    want[1::4] = 1 + 2 * weight[1::4, 1::2].argmax(1)
    want[2::4] = -1
    assert torch.equal(token.long(), want)


def test_logits_of_repeated_biases_the_last_counts():
    x = np.zeros((2, 100), np.float32)
    biases = [[(5, 1.0), (6, 2.0), (5, -3.0), (5, 0.5)], [(99, 4.0)] * 600 + [(99, -4.0)]]
    out, token = logits_case((x, np.ones((2, 3)), None, biases, None, None))
    assert out[0, 5] == 0.5 and out[0, 6] == 2.0 and out[1, 99] == -4.0 and token.tolist() == [6, 0]


def test_logits_ties_masks_and_not_numbers():
    v = 2500
    x = np.full((8, v), -1.0, np.float32)
    x[0, [3, 700, 2000]] = 5.0                       # the lowest of equal ones, across slices
    x[1, :] = np.nan
    x[2, :] = np.nan
    x[2, 1234] = -8.0
    x[3, :] = -np.inf
    x[4, 17] = np.inf
    x[4, 18] = np.nan
    x[5, :] = -3.402823466e38
    x[6, 4] = -0.0
    x[6, 2] = 0.0
    mask = np.zeros((2, (v + 31) // 32), np.uint32)
    mask[1, 2400 // 32] = 1 << (2400 % 32)
    mask_row = np.array([-1, -1, -1, -1, -1, -1, -1, 0], np.int32)
    histories = [[]] * 6 + [[2, 4, 4], []]
    pen = np.array([[1.5, 0.0, 0.0]] * 8)
    out, token = logits_case((x, pen, histories, None, mask, mask_row))
    assert token.tolist() == [3, -1, 1234, -1, 17, 0, 2, -1]
    _, token = logits_case((x, pen, histories, None, mask, np.full(8, 1, np.int32)))
    assert token.tolist() == [2400, -1, -1, -1, 2400, 2400, 2400, 2400]


def test_logits_captured_on_another_stream():
    torch = torch_cuda()
    m, v = 3, 5000
    x, penalty, _, _, mask, mask_row = logits_inputs(m, v, seed=33)
    need = mz.mz_logits_rules_workspace_bytes(m, v)
    ws = torch.full((need // 4,), float("nan"), device="cuda")
    history, off = torch.zeros(1000, device="cuda", dtype=torch.int32), torch.zeros(m + 1, device="cuda", dtype=torch.int64)
    d = [dev(x), dev(penalty), dev(mask.view(np.int32)), dev(mask_row)]
    out, token = torch.zeros(m, v, device="cuda"), torch.zeros(m, device="cuda", dtype=torch.int32)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        mz.mz_logits_rules(d[0].data_ptr(), m, v, v, out.data_ptr(), token.data_ptr(), ws.data_ptr(), need, stream(),
                           penalty_ptr=d[1].data_ptr(), history_ptr=history.data_ptr(), history_off_ptr=off.data_ptr(),
                           mask_ptr=d[2].data_ptr(), n_masks=mask.shape[0], mask_words=mask.shape[1], mask_row_ptr=d[3].data_ptr())
    rng = np.random.default_rng(34)
    for step in range(4):
        x = (rng.standard_normal((m, v)) * 3).astype(np.float32)
        histories = [[int(t) for t in rng.integers(0, 60, 100 * step)] for _ in range(m)]
        flat, offs = rows_of(histories, np.int32)
        d[0].copy_(dev(x)), off.copy_(dev(offs)), history[:len(flat)].copy_(dev(flat))
        g.replay()
        torch.cuda.synchronize()
        ref, bound = logits_oracle(x, penalty, histories, [[]] * m, mask, mask_row)
        close(out, ref, bound, f"step {step}")
        assert np.array_equal(token.cpu().numpy(), picked(out.cpu().numpy()))


# ----------------------------------------------------------------------------- rules on a context's tokens

def tiny_engine(extra=16):
    from paper_2609_01338_amd import workloads as W
    torch_cuda()
    w = W.WORKLOADS["tiny"]
    return w.model, W.make_tokens(w)[0], mz.Engine(w.model, W.make_blob(w), max_ctx=w.n_ctx + extra)


def words_of(allowed, vocab):
    bits = np.zeros((vocab + 31) // 32 * 32, np.uint8)
    bits[list(allowed)] = 1
    return np.packbits(bits, bitorder="little").view(np.uint32)


def test_token_rules_of_a_context():
    """The first token and its logits after the rules, from the logits without them and the context as history."""
    m, ctx, eng = tiny_engine()
    bias = [(5, 2.5), (17, -1.0), (5, 0.75)]
    mask = words_of(set(range(0, m.vocab, 2)) | {5, 17}, m.vocab)
    with eng:
        e = eng.ctx
        mz.mz_prefill_context(e, ctx)
        plain, raw = mz.mz_first_token(e, m.vocab)
        for rules in (dict(repetition=1.3, frequency=0.2, presence=0.1), dict(bias=bias), dict(mask=mask),
                      dict(repetition=0.7, frequency=-0.1, bias=bias, mask=mask)):
            mz.mz_set_token_rules(e, **rules)
            mz.mz_prefill_context(e, ctx)
            tok, logits = mz.mz_first_token(e, m.vocab)
            pen = [[rules.get("repetition", 1.0), rules.get("frequency", 0.0), rules.get("presence", 0.0)]]
            got_mask = rules.get("mask")
            ref, bound = logits_oracle(raw[None], np.array(pen, np.float32), [ctx.tolist()],
                                       [[(t, float(np.float32(v))) for t, v in rules.get("bias", [])]],
                                       None if got_mask is None else got_mask[None], [0])
            close(logits[None], ref, bound, "logits after " + ", ".join(rules))
            assert tok == picked(logits[None])[0]
            mz.mz_prefill_context(e, ctx)
            assert mz.mz_first_token(e) == tok, "without the logits"
        mz.mz_clear_token_rules(e)
        mz.mz_prefill_context(e, ctx)
        again, logits = mz.mz_first_token(e, m.vocab)
        assert again == plain and logits.tobytes() == raw.tobytes()


def test_token_rules_while_generating():
    """The history grows with each token; mz_generate and single steps choose the same; a context cut back
    and continued otherwise counts its own tokens only."""
    m, ctx, eng = tiny_engine()
    with eng:
        e = eng.ctx
        mz.mz_set_token_rules(e, presence=1000.0)
        mz.mz_prefill_context(e, ctx)
        first = mz.mz_first_token(e)
        toks = mz.mz_generate(e, first, 10).tolist()
        seen = ctx.tolist() + [first] + toks
        assert len(set([first] + toks)) == 11 and not set([first] + toks) & set(ctx.tolist())
        mz.mz_truncate_context(e, ctx.size)
        t, steps = first, []
        for _ in range(10):
            mz.mz_restore_and_prefill(e, np.array([t], np.int32))
            t = mz.mz_first_token(e)
            steps.append(t)
        assert steps == toks
        # cut back, then on with a token that was not there before: those cut off may come again
        mz.mz_truncate_context(e, ctx.size)
        other = next(v for v in range(m.vocab) if v not in seen)
        mz.mz_restore_and_prefill(e, np.array([other], np.int32))
        _, logits = mz.mz_first_token(e, m.vocab)
        low = np.nonzero(logits < -500)[0]
        assert set(low.tolist()) == set(ctx.tolist()) | {other}
        # a grammar of five tokens
        allowed = [3, 77, 500, 777, m.vocab - 1]
        mz.mz_set_token_rules(e, mask=words_of(allowed, m.vocab))
        mz.mz_prefill_context(e, ctx)
        toks = mz.mz_generate(e, mz.mz_first_token(e), 6)
        assert set(toks.tolist()) <= set(allowed)


def test_token_rules_that_leave_no_token():
    m, ctx, eng = tiny_engine()
    with eng:
        e = eng.ctx
        mz.mz_set_token_rules(e, mask=words_of([9], m.vocab), bias=[(9, float("-inf"))])
        mz.mz_prefill_context(e, ctx)
        with pytest.raises(mz.MzError) as err:
            mz.mz_first_token(e)
        assert err.value.status == mz.MZ_ESTATE and "rules" in str(err.value)
        with pytest.raises(mz.MzError) as err:
            mz.mz_generate(e, 1, 4)
        assert err.value.status == mz.MZ_ESTATE
        mz.mz_clear_token_rules(e)
        mz.mz_restore_and_prefill(e, np.array([2], np.int32))
        assert 0 <= mz.mz_first_token(e) < m.vocab


def test_token_rules_that_left_no_token_may_be_relaxed():
    """The prefill is not used up: other rules, or none, choose from the same logits, after a step of mz_generate too."""
    m, ctx, eng = tiny_engine()
    with eng:
        e = eng.ctx
        mz.mz_prefill_context(e, ctx)
        plain, raw = mz.mz_first_token(e, m.vocab)
        none = dict(mask=words_of([9], m.vocab), bias=[(9, float("-inf"))])
        for after in ("prefill", "generate"):
            mz.mz_set_token_rules(e, **none)
            if after == "prefill":
                mz.mz_prefill_context(e, ctx)
                call = lambda: mz.mz_first_token(e)                     # noqa: E731
            else:
                mz.mz_truncate_context(e, ctx.size - 1)
                call = lambda: mz.mz_generate(e, int(ctx[-1]), 3)       # noqa: E731
            with pytest.raises(mz.MzError) as err:
                call()
            assert err.value.status == mz.MZ_ESTATE and "rules" in str(err.value)
            with pytest.raises(mz.MzError) as err:                  # and once more under the same
                mz.mz_first_token(e)
            assert err.value.status == mz.MZ_ESTATE and "rules" in str(err.value)
            if after == "prefill":
                mz.mz_clear_token_rules(e)
                tok, logits = mz.mz_first_token(e, m.vocab)
                assert tok == plain and logits.tobytes() == raw.tobytes()
            else:
                mz.mz_set_token_rules(e, mask=words_of([9, 11], m.vocab))
                tok = mz.mz_first_token(e)
                assert tok in (9, 11)
            with pytest.raises(mz.MzError) as err:                  # a chosen token uses it up
                mz.mz_first_token(e)
            assert err.value.status == mz.MZ_ESTATE and "no prefill" in str(err.value)


def test_token_rules_refusals_keep_the_rules():
    m, ctx, eng = tiny_engine()
    nan, inf = float("nan"), float("inf")
    with eng:
        e = eng.ctx
        mz.mz_set_token_rules(e, mask=words_of([9, 10], m.vocab))
        past = words_of([9], m.vocab) * np.uint32(0)
        for bad in (dict(repetition=0.0), dict(repetition=-1.0), dict(repetition=nan), dict(repetition=inf), dict(frequency=inf),
                    dict(presence=nan), dict(bias=[(-1, 0.0)]), dict(bias=[(m.vocab, 0.0)]), dict(bias=[(0, nan)]),
                    dict(bias=[(0, 0.0)] * (m.vocab + 1)), dict(mask=past)):
            with pytest.raises(mz.MzError) as err:
                mz.mz_set_token_rules(e, **bad)
            assert err.value.status == mz.MZ_EINVAL, bad
        mz.mz_prefill_context(e, ctx)
        assert mz.mz_first_token(e) in (9, 10)


def test_token_rules_over_what_was_chosen():
    """history_from leaves the prompt out, whatever its length; past the end of the context nothing counts yet."""
    m, ctx, eng = tiny_engine()
    with eng:
        e = eng.ctx
        mz.mz_prefill_context(e, ctx)
        plain, raw = mz.mz_first_token(e, m.vocab)
        pen = np.array([[1.5, 40.0, 3.0]], np.float32)
        for at in (0, 1, 5, ctx.size - 1, ctx.size, ctx.size + 1, (1 << 31) - 1):
            mz.mz_set_token_rules(e, 1.5, 40.0, 3.0, history_from=at)
            mz.mz_prefill_context(e, ctx)
            tok, logits = mz.mz_first_token(e, m.vocab)
            ref, bound = logits_oracle(raw[None], pen, [ctx[at:].tolist()], [[]], None, [0])
            close(logits[None], ref, bound, f"from {at}")
            assert tok == picked(logits[None])[0]
        # the answer's tokens count as they come, also by mz_generate and after a cut that leaves fewer than at
        mz.mz_set_token_rules(e, presence=1000.0, history_from=ctx.size)
        mz.mz_prefill_context(e, ctx)
        first = mz.mz_first_token(e, m.vocab)[0]
        assert first == plain
        toks = [first] + mz.mz_generate(e, first, 8).tolist()
        assert len(set(toks)) == 9
        mz.mz_truncate_context(e, ctx.size - 1)
        mz.mz_restore_and_prefill(e, ctx[-1:])
        tok, logits = mz.mz_first_token(e, m.vocab)
        assert not (logits < -500).any()
        with pytest.raises(mz.MzError) as err:
            mz.mz_set_token_rules(e, history_from=-1)
        assert err.value.status == mz.MZ_EINVAL


def test_token_rules_of_a_short_mask():
    """The binding refuses a mask that ends before the vocabulary; the rules stay."""
    m, ctx, eng = tiny_engine()
    with eng:
        e = eng.ctx
        mz.mz_set_token_rules(e, mask=words_of([9, 10], m.vocab))
        for words in (0, 1, (m.vocab + 31) // 32 - 1):
            with pytest.raises(mz.MzError) as err:
                mz.mz_set_token_rules(e, mask=np.ones(words, np.uint32))
            assert err.value.status == mz.MZ_EINVAL and "vocabulary" in str(err.value)
        mz.mz_prefill_context(e, ctx)
        assert mz.mz_first_token(e) in (9, 10)


# ----------------------------------------------------------------------------- the calls together

def test_decode_steps_of_a_batch_in_one_graph():
    """Prompts of five requests, then decode steps of all of them, captured once: shared Q4_0 projections with each
    request's adapter, the append, the attention, the output projection, the head and the rules.  Every call's output
    is checked from the buffers that it read; lengths, positions, histories and adapters change between replays."""
    from paper_2609_01338_amd import workloads as W
    torch = torch_cuda()
    nq, nkv, hd, d, V, C, n_seq, R, na = 4, 2, 64, 256, 1024, 16, 5, 16, 3
    dq, dkv, wide = nq * hd, nkv * hd, (nq + 2 * nkv) * hd
    rng = np.random.default_rng(50)
    pack = lambda n, k: dev(mz.mz_q4_gemm_pack(W.encode_q4_0((rng.standard_normal((n, k)) * 0.05).astype(np.float32)), n, k))  # noqa: E731
    w_qkv, w_o, w_lm = pack(wide, d), pack(d, dq), pack(V, d)
    lora = {k: [(rng.standard_normal(s) * 0.1).astype(np.float16) for s in ((na, R, i), (na, o, R))]
            for k, i, o in (("qkv", d, wide), ("o", dq, d))}
    d_lora = {k: [dev(t) for t in v] for k, v in lora.items()}
    rank, scale = np.array([16, 5, 8], np.int32), np.array([1.0, 0.5, 2.0], np.float32)
    d_rank, d_scale = dev(rank), dev(scale)
    n_table, n_rope = 8, 128
    table = rng.permutation(n_seq * n_table).reshape(n_seq, n_table).astype(np.int32)
    rope = rope_table(n_rope, hd)
    d_table, d_rope = dev(table), dev(rope)
    slab = torch.full((n_seq * n_table, 2 * C * dkv), float("nan"), device="cuda", dtype=torch.float16)

    def buffers(m):
        z = lambda *s, dt=torch.float32: torch.zeros(*s, device="cuda", dtype=dt)  # noqa: E731
        h16, i32 = torch.float16, torch.int32
        return dict(m=m, h=z(m, d), x=z(m, d, dt=h16), qkv0=z(m, wide), qkv=z(m, wide), q=z(m, dq, dt=h16), o0=z(m, d), o=z(m, d),
                    att=z(m, dq, dt=h16), logits=z(m, V), out=z(m, V), seq=z(m, dt=i32), pos=z(m, dt=i32), lens=z(m, dt=i32),
                    adapter=z(m, dt=i32), token=z(m, dt=i32), history=z(2000, dt=i32), off=z(m + 1, dt=torch.int64),
                    pen=dev(np.tile(np.array([1.2, 0.1, 0.3], np.float32), (m, 1))), ws=z(8 << 20, dt=torch.uint8))

    def project(b, x, k, w, n, y):
        mz.mz_q4_gemm_ex(x.data_ptr(), b["m"], n, k, w.data_ptr(), 0, y.data_ptr(), stream())

    def adapt(b, name, x, k, n, base, y):
        a, bb = d_lora[name]
        mz.mz_lora_add(x.data_ptr(), b["m"], k, b["adapter"].data_ptr(), na, a.data_ptr(), bb.data_ptr(), R, n, base.data_ptr(),
                       y.data_ptr(), y.shape[1], b["ws"].data_ptr(), b["ws"].numel(), stream(), scale_ptr=d_scale.data_ptr(),
                       rank_ptr=d_rank.data_ptr())

    def to_chunks(b):
        mz.mz_rmsnorm(b["h"].data_ptr(), b["m"], d, 1e-5, b["x"].data_ptr(), stream())
        project(b, b["x"], d, w_qkv, wide, b["qkv0"])
        adapt(b, "qkv", b["x"], d, wide, b["qkv0"], b["qkv"])
        p = b["qkv"].data_ptr()
        mz.mz_kv_append(b["m"], p + dq * 4, p + (dq + dkv) * 4, b["seq"].data_ptr(), b["pos"].data_ptr(), d_rope.data_ptr(), n_rope,
                        slab.data_ptr(), n_seq * n_table, d_table.data_ptr(), n_seq, n_table, C, nkv, hd, stream(), q_ptr=p, n_q=nq,
                        q_out_ptr=b["q"].data_ptr(), k_stride=wide, v_stride=wide, q_stride=wide)

    def step(b):
        to_chunks(b)
        mz.mz_attention_batch(b["q"].data_ptr(), b["lens"].data_ptr(), n_seq, slab.data_ptr(), n_seq * n_table, d_table.data_ptr(),
                              n_table, C, nq, nkv, hd, b["ws"].data_ptr(), b["ws"].numel(), b["att"].data_ptr(), stream())
        project(b, b["att"], dq, w_o, d, b["o0"])
        adapt(b, "o", b["att"], dq, d, b["o0"], b["o"])
        mz.mz_rmsnorm(b["o"].data_ptr(), b["m"], d, 1e-5, b["x"].data_ptr(), stream())
        project(b, b["x"], d, w_lm, V, b["logits"])
        mz.mz_logits_rules(b["logits"].data_ptr(), b["m"], V, V, b["out"].data_ptr(), b["token"].data_ptr(), b["ws"].data_ptr(),
                           b["ws"].numel(), stream(), penalty_ptr=b["pen"].data_ptr(), history_ptr=b["history"].data_ptr(),
                           history_off_ptr=b["off"].data_ptr())

    host = lambda t: t.cpu().numpy()  # noqa: E731

    def check_chunks(b, before, adapter, what):
        base, x = host(b["qkv0"]), host(b["x_qkv"])
        ref, bound = lora_oracle(x, adapter, *lora["qkv"], scale, rank, base, wide)
        close(b["qkv"], ref, bound, what + ": adapters")
        q, k, v = np.split(host(b["qkv"]), [dq, dq + dkv], 1)
        ref, bound, qr, qb, wrote = append_oracle(k, v, q, host(b["seq"]), host(b["pos"]), rope, before, table, C, nkv, hd)
        close(slab, ref, bound, what + ": chunks")
        close(b["q"][dev(wrote)], qr[wrote], qb[wrote], what + ": queries")

    # the prompts, of uneven lengths, and three rows of padding
    lens = np.array([33, 1, 16, 90, 47], np.int32)
    p = buffers(int(lens.sum()) + 3)
    seq = np.concatenate([np.repeat(np.arange(n_seq), lens), [-1] * 3]).astype(np.int32)
    pos = np.concatenate([np.arange(n) for n in lens] + [[0] * 3]).astype(np.int32)
    adapter = np.where(seq >= 0, np.array([0, 1, -1, 2, 1])[seq], -1).astype(np.int32)
    for name, t in (("h", rng.standard_normal((len(seq), d)).astype(np.float32)), ("seq", seq), ("pos", pos), ("adapter", adapter)):
        p[name].copy_(dev(t))
    before = host(slab)
    to_chunks(p)
    torch.cuda.synchronize()
    p["x_qkv"] = p["x"]
    check_chunks(p, before, adapter, "prompts")
    # decode steps
    b = buffers(n_seq)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        step(b)
    histories = [[int(t) for t in rng.integers(0, V, n)] for n in lens]
    for i in range(4):
        lens = lens + 1
        adapter = np.array([[0, 1, -1, 2, 1], [2, 2, 2, 2, 2], [-1] * 5, [1, 0, 2, 5, 0]][i], np.int32)
        flat, off = rows_of(histories, np.int32)
        for name, t in (("h", rng.standard_normal((n_seq, d)).astype(np.float32)), ("seq", np.arange(n_seq, dtype=np.int32)),
                        ("pos", lens - 1), ("lens", lens), ("adapter", adapter), ("off", off)):
            b[name].copy_(dev(t))
        b["history"][:len(flat)].copy_(dev(flat))
        before = host(slab)
        g.replay()
        torch.cuda.synchronize()
        x = torch.zeros(n_seq, d, device="cuda", dtype=torch.float16)      # the step's x, which the head's took the place of
        mz.mz_rmsnorm(b["h"].data_ptr(), n_seq, d, 1e-5, x.data_ptr(), stream())
        b["x_qkv"] = x
        check_chunks(b, before, adapter, f"step {i}")
        ref, bound = attention_oracle(host(b["q"]), lens, host(slab), table, C, nq, nkv, hd)
        close(b["att"], ref, bound, f"step {i}: attention")
        ref, bound = lora_oracle(host(b["att"]), adapter, *lora["o"], scale, rank, host(b["o0"]), d)
        close(b["o"], ref, bound, f"step {i}: output adapters")
        ref, bound = logits_oracle(host(b["logits"]), host(b["pen"]), histories, [[]] * n_seq, None, None)
        close(b["out"], ref, bound, f"step {i}: logits")
        assert np.array_equal(host(b["token"]), picked(host(b["out"])))
        for s, t in enumerate(host(b["token"]).tolist()):
            histories[s].append(t)
