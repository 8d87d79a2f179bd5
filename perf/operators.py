"""The operators of a batched decode step: what they compute, in plain form, and what is timed.

Where ``mz_ctx`` restores and continues one cached context, these kernel-level calls carry one step of
many requests at once over the same Q4_0 weights and the same chunked KV slab:

* ``append``: the step's keys and values rotated to their positions and written into the chunks of
  their sequences, and the queries rotated beside them (``mz_kv_append``);
* ``attention``: one new token of every sequence against its cached chunks (``mz_attention_batch``);
* ``lora``: every row's own low-rank adapter added to a shared projection (``mz_lora_add``);
* ``logits``: penalties for repeated tokens, biases and grammar masks on the rows' logits, and the
  token each row takes (``mz_logits_rules``).

Slots are laid out as for ``mz_attention``: keys [chunk][n_kv * head_dim], then values
[n_kv * head_dim][chunk], in halves.  Shapes are those of the framework's model classes.
"""

import itertools
import math
import random

import torch

own = False

# d_model, query heads, key/value heads, head dimension, MLP width, vocabulary, rotary base
MODELS = {"tiny": (256, 4, 2, 64, 688, 1024, 1e4), "1b": (2048, 32, 8, 64, 8192, 128256, 5e5),
          "1p5b": (1536, 12, 2, 128, 8960, 151936, 5e5), "8b": (4096, 32, 8, 128, 14336, 128256, 5e5)}


# ----------------------------------------------------------------------------- the cases

def listed():
    return [
        # one request's token on the 1B class: the smallest call, all latency
        dict(name="append_1b_1row", kind="append", model="1b", seqs=1, rows=1, past=777, chunk=256, f32=True, mix=1),
        # a decode step of 64 requests on the 8B class, from the projections' fp32 rows
        dict(name="append_8b_64rows", kind="append", model="8b", seqs=64, rows=64, past=16384, chunk=256, f32=True,
             mix=2),
        # the prompts of five requests joined in one prefill, of uneven lengths, f16 projections
        dict(name="append_8b_prompts", kind="append", model="8b", seqs=5, rows=4099, past=3000, chunk=256, f32=False,
             mix=3),
        # one chat on the 1B class
        dict(name="attn_1b_1x2048", kind="attention", model="1b", seqs=1, ctx=2048, even=True, chunk=256, mix=4),
        # eight requests of uneven lengths, small pages, a query group that is no power of two
        dict(name="attn_1p5b_8_ragged", kind="attention", model="1p5b", seqs=8, ctx=16384, even=False, chunk=16, mix=5),
        # one long document on the 8B class
        dict(name="attn_8b_1x32768", kind="attention", model="8b", seqs=1, ctx=32768, even=True, chunk=256, mix=6),
        # a full batch of uneven lengths
        dict(name="attn_8b_64_ragged", kind="attention", model="8b", seqs=64, ctx=8192, even=False, chunk=256, mix=7),
        # one request's adapter beside the query projection
        dict(name="lora_1b_1row", kind="lora", model="1b", proj="q", rows=1, adapters=4, rank=16, runs=False, mix=8),
        # a decode step of 33 requests over 24 adapters of mixed ranks, some requests without one
        dict(name="lora_8b_33rows", kind="lora", model="8b", proj="o", rows=33, adapters=24, rank=32, runs=False,
             mix=9),
        # prompts of six requests in one prefill, each with its adapter
        dict(name="lora_8b_prompts", kind="lora", model="8b", proj="q", rows=4099, adapters=6, rank=64, runs=True,
             mix=10),
        # one request: penalties over its context, a few biases, a grammar
        dict(name="logits_8b_1row", kind="logits", vocab=128256, rows=1, history=2048, biases=16, masks=1, mix=11),
        # a full batch with long histories
        dict(name="logits_1p5b_64rows", kind="logits", vocab=151936, rows=64, history=4096, biases=300, masks=8, mix=12),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "lora", "lora", "logits"])
    model = rng.choice(["tiny", "1b", "1p5b", "8b"])
    mix = rng.randrange(100, 1 << 30)
    if kind == "append":
        rows = _log(rng, 1, 4096)
        seqs = rows if rows <= 96 and rng.random() < 0.5 else rng.randint(1, min(rows, 8))
        return dict(kind=kind, model=model, seqs=seqs, rows=rows, past=_log(rng, 1, 16384),
                    chunk=rng.choice([16, 64, 256]), f32=rng.random() < 0.5, mix=mix)
    if kind == "attention":
        seqs = _log(rng, 1, 64)
        ctx = _log(rng, 1, min(32768, 8192 * 48 // seqs))
        return dict(kind=kind, model=model, seqs=seqs, ctx=ctx, even=seqs * ctx <= 128 * 1024 and rng.random() < 0.5,
                    chunk=rng.choice([8, 16, 64, 256]), mix=mix)
    if kind == "lora":
        rows = _log(rng, 1, 4096)
        return dict(kind=kind, model=model, proj=rng.choice(["q", "kv", "o"] + ["down"] * (rows <= 1024)), rows=rows,
                    adapters=rng.randint(1, 32 if rows <= 256 else 6), rank=rng.choice([8, 16, 32, 64]),
                    runs=rows > 256 or rng.random() < 0.5, mix=mix)
    return dict(kind=kind, vocab=MODELS[model][5] - rng.choice([0, 0, rng.randint(1, 99)]), rows=_log(rng, 1, 64),
                history=_log(rng, 1, 8192), biases=_log(rng, 1, 300), masks=rng.randint(1, 8), mix=mix)


def _lens(case):
    """Cached tokens of every sequence: all of them ctx, or spread over its lower sixteenth part and up."""
    r, ctx = random.Random(case["mix"]), case["ctx"]
    return [ctx if case["even"] or i == 0 else _log(r, max(1, ctx // 16), ctx) for i in range(case["seqs"])]


def _spans(case):
    """(first position, rows) of every sequence of an append."""
    r, n, rows = random.Random(case["mix"]), case["seqs"], case["rows"]
    cuts = [0] + sorted(r.sample(range(1, rows), n - 1)) + [rows]
    return [(r.randint(0, case["past"]), b - a) for a, b in zip(cuts, cuts[1:])]


def _adapter_rows(case):
    """The adapter of every row (-1: none): requests one after the other, or every row a request of its own."""
    r, n, rows = random.Random(case["mix"]), case["adapters"], case["rows"]
    if not case["runs"]:
        return [r.randrange(n) if rows == 1 or r.random() < 0.9 else -1 for _ in range(rows)]
    k = min(rows, n)
    cuts = [0] + sorted(r.sample(range(1, rows), k - 1)) + [rows]
    return [i for i, (a, b) in enumerate(zip(cuts, cuts[1:])) for _ in range(b - a)]


def _ranks(case):
    r = random.Random(case["mix"] + 1)
    return [max(1, case["rank"] >> r.choice([0, 0, 1, 2])) for _ in range(case["adapters"])]


def _projection(case):
    d, nq, nkv, hd, ff = MODELS[case["model"]][:5]
    return {"q": (d, nq * hd), "kv": (d, 2 * nkv * hd), "o": (nq * hd, d), "down": ((ff + 127) // 128 * 128, d)}[case["proj"]]


def _histories(case):
    r = random.Random(case["mix"])
    return [case["history"] if i == 0 else r.randint(0, case["history"]) for i in range(case["rows"])]


# ----------------------------------------------------------------------------- inputs

def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + salt) % (1 << 62))


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _tables(g, n_chunks):
    """A chunk table whose chunks lie anywhere in the slab, -1 where a sequence has no chunk."""
    wide, total = max(n_chunks), sum(n_chunks)
    table = torch.full((len(n_chunks), wide), -1, dtype=torch.int32, device="cuda")
    held = torch.arange(wide, device="cuda")[None, :] < _ints(n_chunks)[:, None]
    table[held] = torch.randperm(total, device="cuda", generator=g).int()
    return table, total


def _prepare_append(case, seed):
    d, nq, nkv, hd, _, _, theta = MODELS[case["model"]]
    g, c = _gen(seed, 1), case["chunk"]
    spans = _spans(case)
    pos = [p + i for p, n in spans for i in range(n)]
    seq = [s for s, (_, n) in enumerate(spans) for _ in range(n)]
    # chunks of the sequences' whole pasts are in the table; those that the step does not touch share slot 0
    table = torch.zeros(len(spans), max(p + n - 1 for p, n in spans) // c + 1, dtype=torch.int32, device="cuda")
    touched = sorted({(s, p // c) for s, p in zip(seq, pos)})
    at = _ints(touched, torch.int64)
    table[at[:, 0], at[:, 1]] = 1 + torch.randperm(len(touched), device="cuda", generator=g).int()
    n_slots = len(touched) + 1
    n_rope = max(pos) + 1
    inv = theta ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)
    ang = torch.arange(n_rope, device="cuda", dtype=torch.float64)[:, None] * inv[None, :]
    # one row holds the step's queries, keys and values, as a fused projection leaves them
    qkv = torch.randn(case["rows"], (nq + 2 * nkv) * hd, device="cuda", generator=g)
    return dict(kind="append", nq=nq, nkv=nkv, hd=hd, c=c, m=case["rows"], f32=case["f32"],
                qkv=qkv if case["f32"] else qkv.half(), seq=_ints(seq), pos=_ints(pos), n_seq=len(spans),
                table=table, n_slots=n_slots, n_rope=n_rope,
                rope=torch.stack([ang.cos(), ang.sin()], 2).float().contiguous(),
                slab=torch.randn(n_slots, 2 * c * nkv * hd, device="cuda", generator=g).half(),
                q_out=torch.zeros(case["rows"], nq * hd, device="cuda", dtype=torch.float16))


def _prepare_attention(case, seed):
    _, nq, nkv, hd, _, _, _ = MODELS[case["model"]]
    g, c, lens = _gen(seed, 2), case["chunk"], _lens(case)
    table, n_slots = _tables(g, [(n + c - 1) // c for n in lens])
    q = torch.randn(len(lens), nq * hd, device="cuda", generator=g).half()
    slab = torch.empty(n_slots, 2 * c * nkv * hd, device="cuda", dtype=torch.float16).normal_(generator=g)
    ws = torch.empty(64 << 20, device="cuda", dtype=torch.uint8)
    return dict(kind="attention", nq=nq, nkv=nkv, hd=hd, c=c, m=len(lens), q=q, slab=slab, n_slots=n_slots,
                table=table, lens=_ints(lens), ws=ws, out=torch.zeros_like(q))


def _prepare_lora(case, seed):
    g, (k, n), r, na = _gen(seed, 3), _projection(case), case["rank"], case["adapters"]
    x = torch.randn(case["rows"], k, device="cuda", generator=g).half()
    a = (torch.randn(na, r, k, device="cuda", generator=g) / math.sqrt(k)).half()
    b = (torch.randn(na, n, r, device="cuda", generator=g) * 0.1).half()
    base = torch.randn(case["rows"], (n + 255) // 256 * 256, device="cuda", generator=g)
    return dict(kind="lora", m=case["rows"], k=k, n=n, r=r, na=na, x=x, a=a, b=b, base=base, y=torch.zeros_like(base),
                scale=torch.rand(na, device="cuda", generator=g) + 0.5, rank=_ints(_ranks(case)),
                adapter=_ints(_adapter_rows(case)), ws=torch.empty(64 << 20, device="cuda", dtype=torch.uint8))


def _prepare_logits(case, seed):
    g, m, v = _gen(seed, 4), case["rows"], case["vocab"]
    offsets = list(itertools.accumulate(_histories(case), initial=0))
    total = offsets[-1]
    # frequent tokens are the low ones, so histories repeat them; the biases name tokens anywhere
    history = (torch.rand(total, device="cuda", generator=g) ** 3 * v).int().clamp_(max=v - 1)
    logits = torch.randn(m, v, device="cuda", generator=g) * 3
    penalty = torch.rand(m, 3, device="cuda", generator=g)
    penalty[:, 0] += 1.0
    words = (v + 31) // 32
    mask = torch.randint(-(1 << 31), 1 << 31, (case["masks"], words), device="cuda", generator=g).int()
    rows = random.Random(case["mix"] + 2)
    return dict(kind="logits", m=m, v=v, words=words, logits=logits, out=torch.zeros_like(logits), penalty=penalty,
                history=history, history_off=_ints(offsets, torch.int64),
                bias_token=torch.randint(0, v, (m * case["biases"],), device="cuda", generator=g).int(),
                bias_value=torch.randn(m * case["biases"], device="cuda", generator=g) * 2,
                bias_off=_ints([i * case["biases"] for i in range(m + 1)], torch.int64),
                mask=mask, n_masks=case["masks"], mask_row=_ints([rows.randint(-1, case["masks"] - 1) for _ in range(m)]),
                token=torch.zeros(m, device="cuda", dtype=torch.int32),
                ws=torch.empty(1 << 20, device="cuda", dtype=torch.uint8))


def prepare(case, seed):
    return {"append": _prepare_append, "attention": _prepare_attention, "lora": _prepare_lora,
            "logits": _prepare_logits}[case["kind"]](case, seed)


# ----------------------------------------------------------------------------- the calls of the framework

def _own_append(s):
    from paper_2609_01338_amd import mz
    q, size = s["qkv"].data_ptr(), 4 if s["f32"] else 2
    wide, dq, dkv = s["qkv"].shape[1], s["nq"] * s["hd"], s["nkv"] * s["hd"]
    mz.mz_kv_append(s["m"], q + dq * size, q + (dq + dkv) * size, s["seq"].data_ptr(), s["pos"].data_ptr(),
                    s["rope"].data_ptr(), s["n_rope"], s["slab"].data_ptr(), s["n_slots"], s["table"].data_ptr(),
                    s["n_seq"], s["table"].shape[1], s["c"], s["nkv"], s["hd"],
                    torch.cuda.current_stream().cuda_stream, q_ptr=q, n_q=s["nq"], q_out_ptr=s["q_out"].data_ptr(),
                    k_stride=wide, v_stride=wide, q_stride=wide, f32=s["f32"])
    return {"slab": s["slab"], "q": s["q_out"]}


def _own_attention(s):
    from paper_2609_01338_amd import mz
    mz.mz_attention_batch(s["q"].data_ptr(), s["lens"].data_ptr(), s["m"], s["slab"].data_ptr(), s["n_slots"],
                          s["table"].data_ptr(), s["table"].shape[1], s["c"], s["nq"], s["nkv"], s["hd"],
                          s["ws"].data_ptr(), s["ws"].numel(), s["out"].data_ptr(),
                          torch.cuda.current_stream().cuda_stream)
    return s["out"]


def _own_lora(s):
    from paper_2609_01338_amd import mz
    mz.mz_lora_add(s["x"].data_ptr(), s["m"], s["k"], s["adapter"].data_ptr(), s["na"], s["a"].data_ptr(),
                   s["b"].data_ptr(), s["r"], s["n"], s["base"].data_ptr(), s["y"].data_ptr(), s["y"].shape[1],
                   s["ws"].data_ptr(), s["ws"].numel(), torch.cuda.current_stream().cuda_stream,
                   scale_ptr=s["scale"].data_ptr(), rank_ptr=s["rank"].data_ptr())
    return s["y"]


def _own_logits(s):
    from paper_2609_01338_amd import mz
    mz.mz_logits_rules(s["logits"].data_ptr(), s["m"], s["v"], s["v"], s["out"].data_ptr(), s["token"].data_ptr(),
                       s["ws"].data_ptr(), s["ws"].numel(), torch.cuda.current_stream().cuda_stream,
                       penalty_ptr=s["penalty"].data_ptr(), history_ptr=s["history"].data_ptr(),
                       history_off_ptr=s["history_off"].data_ptr(), bias_token_ptr=s["bias_token"].data_ptr(),
                       bias_value_ptr=s["bias_value"].data_ptr(), bias_off_ptr=s["bias_off"].data_ptr(),
                       mask_ptr=s["mask"].data_ptr(), n_masks=s["n_masks"], mask_words=s["words"],
                       mask_row_ptr=s["mask_row"].data_ptr())
    return {"logits": s["out"], "token": s["token"]}


# ----------------------------------------------------------------------------- the plain forms

def _rotated(x, rope):
    """Rotate-half pairs (i, i + head_dim / 2) of x [rows][heads][head_dim] by rope [rows][head_dim / 2][2]."""
    a, b = x.chunk(2, 2)
    c, s = rope[:, None, :, 0], rope[:, None, :, 1]
    return torch.cat([a * c - b * s, b * c + a * s], 2)


def _plain_append(s):
    m, nq, nkv, hd, c = s["m"], s["nq"], s["nkv"], s["hd"], s["c"]
    heads = s["qkv"].float().view(m, nq + 2 * nkv, hd)
    pos, seq = s["pos"].long(), s["seq"].long()
    turned = _rotated(heads[:, :nq + nkv], s["rope"][pos]).half()
    slot, at = s["table"][seq, pos // c].long(), pos % c
    half = s["slab"].view(s["n_slots"], 2, -1)
    half[:, 0].unflatten(1, (c, nkv, hd))[slot, at] = turned[:, nq:]
    half[:, 1].unflatten(1, (nkv, hd, c))[slot, :, :, at] = heads[:, nq + nkv:].half()
    s["q_out"].copy_(turned[:, :nq].reshape(m, -1))
    return {"slab": s["slab"], "q": s["q_out"]}


def _plain_attention(s):
    b, nq, nkv, hd, c = s["m"], s["nq"], s["nkv"], s["hd"], s["c"]
    half = s["slab"].view(s["n_slots"], 2, -1)
    slot = s["table"].long().clamp(min=0)
    top = slot.shape[1] * c
    k = half[:, 0].unflatten(1, (c, nkv, hd))[slot].float().view(b, top, nkv, hd).permute(0, 2, 3, 1).contiguous()
    seen = torch.arange(top, device="cuda")[None, :] < s["lens"][:, None]
    score = torch.matmul(s["q"].float().view(b, nkv, nq // nkv, hd), k) / math.sqrt(hd)
    del k
    score = torch.where(seen[:, None, None, :], score, -math.inf)
    high = score.amax(3, keepdim=True)
    weight = torch.exp(score - torch.where(high == -math.inf, 0.0, high))
    v = half[:, 1].unflatten(1, (nkv, hd, c))[slot].float().permute(0, 2, 1, 4, 3).reshape(b, nkv, top, hd)
    v = torch.where(seen[:, None, :, None], v, 0.0)
    out = torch.matmul(weight, v) / weight.sum(3, keepdim=True)
    s["out"].copy_(torch.where(s["lens"][:, None, None, None] > 0, out, 0.0).reshape(b, -1))
    return s["out"]


def _plain_lora(s):
    m, r, na, n = s["m"], s["r"], s["na"], s["n"]
    ids = torch.arange(na, device="cuda")
    mine = (s["adapter"][:, None] == ids[None, :]).float() * s["scale"][None, :]
    used = (torch.arange(r, device="cuda")[None, :] < s["rank"][:, None]).float()
    low = torch.matmul(s["x"].float(), s["a"].float().view(na * r, -1).T).view(m, na, r)
    low = (low * mine[:, :, None] * used[None]).view(m, na * r)
    s["y"].copy_(s["base"])
    s["y"][:, :n] += torch.matmul(low, s["b"].float().transpose(1, 2).reshape(na * r, n))
    return s["y"]


def _plain_logits(s):
    m, v, x = s["m"], s["v"], s["logits"]
    n = s["history"].numel()
    row = torch.searchsorted(s["history_off"], torch.arange(n, device="cuda"), right=True) - 1
    count = torch.zeros(m * v, device="cuda")
    count.index_add_(0, row * v + s["history"].long(), torch.ones(n, device="cuda"))
    count = count.view(m, v)
    rep, freq, pres = s["penalty"][:, 0:1], s["penalty"][:, 1:2], s["penalty"][:, 2:3]
    held = torch.where(x > 0, x / rep, x * rep) - count * freq - pres
    x = torch.where(count > 0, held, x)
    # of several biases for one token the last counts
    n = s["bias_token"].numel()
    entry = torch.arange(n, device="cuda")
    row = torch.searchsorted(s["bias_off"], entry, right=True) - 1
    last = torch.full((m * v,), -1, dtype=torch.int64, device="cuda")
    last.scatter_reduce_(0, row * v + s["bias_token"].long(), entry, "amax")
    last = last.view(m, v)
    x = torch.where(last >= 0, x + s["bias_value"][last.clamp(min=0)], x)
    ids = torch.arange(v, device="cuda")
    bits = (s["mask"][s["mask_row"].clamp(min=0).long()][:, ids // 32] >> (ids % 32).int()[None, :]) & 1
    x = torch.where((bits == 1) | (s["mask_row"][:, None] < 0), x, -math.inf)
    s["out"].copy_(x)
    best = torch.where(x.isnan(), -math.inf, x)
    top = best.amax(1, keepdim=True)
    first = torch.where(best == top, ids[None, :], v).amin(1, keepdim=True)
    s["token"].copy_(torch.where(top > -math.inf, first, -1)[:, 0])
    return {"logits": s["out"], "token": s["token"]}


def run(state):
    if own:
        return {"append": _own_append, "attention": _own_attention, "lora": _own_lora,
                "logits": _own_logits}[state["kind"]](state)
    return {"append": _plain_append, "attention": _plain_attention, "lora": _plain_lora,
            "logits": _plain_logits}[state["kind"]](state)


# ----------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "logits":
        m, v, lens = case["rows"], case["vocab"], _histories(case)
        return {"bytes": m * v * 8 + case["masks"] * ((v + 31) // 32) * 4 + 4 * sum(lens) + 8 * m * case["biases"],
                "flops": 6.0 * m * v}
    _, nq, nkv, hd, _, _, _ = MODELS[case["model"]]
    if case["kind"] == "append":
        m, wide = case["rows"], (nq + 2 * nkv) * hd
        return {"bytes": m * (wide * ((4 if case["f32"] else 2) + 2) + 4 * hd + 8), "flops": 3.0 * m * (nq + nkv) * hd}
    if case["kind"] == "attention":
        keys = sum(_lens(case))
        return {"bytes": keys * nkv * hd * 4 + case["seqs"] * nq * hd * 4, "flops": 4.0 * keys * nq * hd}
    k, n = _projection(case)
    rows, ranks = _adapter_rows(case), _ranks(case)
    each = sum(ranks[a] for a in set(rows) if a >= 0)
    # x of the rows with an adapter, every used adapter, the projection's rows in and out
    return {"bytes": sum(a >= 0 for a in rows) * k * 2 + each * (k + n) * 2 + len(rows) * n * 8,
            "flops": 2.0 * sum(ranks[a] for a in rows if a >= 0) * (k + n)}


# ----------------------------------------------------------------------------- in 64 bits

def _exact_append(case, seed):
    s = _prepare_append(case, seed)
    nq, nkv, hd, c = s["nq"], s["nkv"], s["hd"], s["c"]
    dq, dkv, h2 = nq * hd, nkv * hd, hd // 2
    x = s["qkv"].double()
    slab = s["slab"].double()
    pos, seq, table = s["pos"].tolist(), s["seq"].tolist(), s["table"].tolist()
    start = torch.tensor([table[b][p // c] * 2 * c * dkv for b, p in zip(seq, pos)], device="cuda")
    at = torch.tensor([p % c for p in pos], device="cuda")
    cs = s["rope"][s["pos"].long()].double()
    flat = slab.view(-1)
    q = torch.empty(s["m"], dq, device="cuda", dtype=torch.float64)
    for head in range(nq + nkv):
        u, w = x[:, head * hd:head * hd + h2], x[:, head * hd + h2:(head + 1) * hd]
        turned = torch.cat([u * cs[:, :, 0] - w * cs[:, :, 1], w * cs[:, :, 0] + u * cs[:, :, 1]], 1)
        if head < nq:
            q[:, head * hd:(head + 1) * hd] = turned
        else:
            to = (start + at * dkv + (head - nq) * hd)[:, None] + torch.arange(hd, device="cuda")[None, :]
            flat[to] = turned
    to = (start + c * dkv + at)[:, None] + c * torch.arange(dkv, device="cuda")[None, :]
    flat[to] = x[:, dq + dkv:]
    return {"slab": slab, "q": q}


def _exact_attention(case, seed):
    s = _prepare_attention(case, seed)
    nq, nkv, hd, c = s["nq"], s["nkv"], s["hd"], s["c"]
    out = torch.zeros(s["m"], nq * hd, device="cuda", dtype=torch.float64)
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        slots = s["slab"][s["table"][b, :(n + c - 1) // c].long()].double()
        keys = slots[:, :c * nkv * hd].reshape(-1, nkv * hd)[:n]
        values = slots[:, c * nkv * hd:].reshape(-1, nkv * hd, c).transpose(1, 2).reshape(-1, nkv * hd)[:n]
        for h in range(nq):
            kv = h // (nq // nkv)
            row = keys[:, kv * hd:(kv + 1) * hd] @ s["q"][b, h * hd:(h + 1) * hd].double() / math.sqrt(hd)
            out[b, h * hd:(h + 1) * hd] = torch.softmax(row, 0) @ values[:, kv * hd:(kv + 1) * hd]
    return out


def _exact_lora(case, seed):
    s = _prepare_lora(case, seed)
    y, ranks = s["base"].double(), s["rank"].tolist()
    for a in range(s["na"]):
        rows = (s["adapter"] == a).nonzero()[:, 0]
        low = s["x"][rows].double() @ s["a"][a, :ranks[a]].double().T
        y[rows, :s["n"]] += s["scale"][a].double() * (low @ s["b"][a, :, :ranks[a]].double().T)
    return y


def _exact_logits(case, seed):
    s = _prepare_logits(case, seed)
    out, token = [], []
    for i in range(s["m"]):
        x = s["logits"][i].double()
        a, b = s["history_off"][i:i + 2].tolist()
        rep, freq, pres = s["penalty"][i].double().tolist()
        ids, count = torch.unique(s["history"][a:b].long(), return_counts=True)
        old = x[ids]
        x[ids] = torch.where(old > 0, old / rep, old * rep) - freq * count - pres
        a, b = s["bias_off"][i:i + 2].tolist()
        bias = dict(zip(s["bias_token"][a:b].tolist(), s["bias_value"][a:b].tolist()))
        x[_ints(list(bias), torch.int64)] += torch.tensor(list(bias.values()), dtype=torch.float64, device="cuda")
        if (k := int(s["mask_row"][i])) >= 0:
            allowed = (s["mask"][k].long()[:, None] >> torch.arange(32, device="cuda")[None, :]) & 1
            x[allowed.view(-1)[:s["v"]] == 0] = -math.inf
        out.append(x)
        token.append(int(torch.argmax(x)))
    return {"logits": torch.stack(out), "token": torch.tensor(token, dtype=torch.int32, device="cuda")}


def exact(case, seed):
    return {"append": _exact_append, "attention": _exact_attention, "lora": _exact_lora,
            "logits": _exact_logits}[case["kind"]](case, seed)
