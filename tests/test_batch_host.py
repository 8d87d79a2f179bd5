"""Refusals of the calls that carry a decode step of many sequences: every one
is found on the host before anything is enqueued, so they need no GPU.  The
device pointers are never followed."""

import os

import pytest

from paper_2609_01338_amd import mz

P = 4096          # stands for a device pointer on a 16-byte boundary


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(mz.LIB_PATH):
        from paper_2609_01338_amd import build
        build.build_all()
    mz.lib()


def refused(fn, *args, match=None, **kw):
    with pytest.raises(mz.MzError) as e:
        fn(*args, **kw)
    assert e.value.status == mz.MZ_EINVAL
    if match:
        assert match in str(e.value), str(e.value)


APPEND = dict(m=3, k_ptr=P, v_ptr=P, seq_ptr=P, pos_ptr=P, rope_cs_ptr=P, n_rope=64, slab_ptr=P, n_slots=4, table_ptr=P,
              n_seq=2, n_table=4, chunk_tokens=16, n_kv=2, head_dim=64, q_ptr=P, n_q=4, q_out_ptr=P)


@pytest.mark.parametrize("bad,match", [
    (dict(m=-1), "negative"),
    (dict(k_ptr=0), "NULL"), (dict(v_ptr=0), "NULL"), (dict(seq_ptr=0), "NULL"), (dict(pos_ptr=0), "NULL"),
    (dict(rope_cs_ptr=0), "NULL"), (dict(slab_ptr=0), "NULL"), (dict(table_ptr=0), "NULL"),
    (dict(q_ptr=0), "q_out"), (dict(q_out_ptr=0), "q_out"),
    (dict(head_dim=48), "head_dim"), (dict(head_dim=256), "head_dim"),
    (dict(n_kv=0), "head"), (dict(n_q=-1), "head"), (dict(n_kv=1025), "head"),
    (dict(n_rope=0), "n_rope"), (dict(n_slots=0), "positive"), (dict(n_seq=0), "positive"), (dict(n_table=0), "positive"),
    (dict(chunk_tokens=4), "chunk_tokens"), (dict(chunk_tokens=24), "chunk_tokens"), (dict(chunk_tokens=-8), "chunk_tokens"),
    (dict(n_table=1 << 27), "2^30"),
    (dict(k_stride=124), "stride"), (dict(v_stride=64), "stride"), (dict(q_stride=-256), "stride"),
    (dict(k_stride=130), "16-byte"), (dict(v_stride=129), "16-byte"), (dict(q_stride=258), "16-byte"),
    (dict(f32=False, k_stride=132), "16-byte"),
    (dict(k_ptr=P + 4), "16-byte"), (dict(v_ptr=P + 8), "16-byte"), (dict(q_ptr=P + 2), "16-byte"),
    (dict(slab_ptr=P + 8), "16-byte"), (dict(rope_cs_ptr=P + 8), "16-byte"), (dict(q_out_ptr=P + 8), "16-byte"),
    (dict(f32=2), "f32"), (dict(m=(1 << 31) - 1, n_q=1024, n_kv=1024, head_dim=128), "too many"),
])
def test_kv_append_refusals(bad, match):
    refused(mz.mz_kv_append, **{**APPEND, **bad}, match=match)


def test_kv_append_no_rows():
    mz.mz_kv_append(**{**APPEND, "m": 0})     # nothing to do, nothing enqueued


ATTENTION = dict(q_ptr=P, lens_ptr=P, n_seq=3, slab_ptr=P, n_slots=8, table_ptr=P, n_table=4, chunk_tokens=16, n_q=8, n_kv=2,
                 head_dim=64, ws_ptr=P, ws_bytes=1 << 30, out_ptr=P)


@pytest.mark.parametrize("bad,match", [
    (dict(q_ptr=0), "NULL"), (dict(lens_ptr=0), "NULL"), (dict(slab_ptr=0), "NULL"), (dict(table_ptr=0), "NULL"),
    (dict(ws_ptr=0), "NULL"), (dict(out_ptr=0), "NULL"),
    (dict(n_seq=0), "positive"), (dict(n_slots=-1), "positive"), (dict(n_table=0), "positive"),
    (dict(chunk_tokens=4), "chunk_tokens"), (dict(chunk_tokens=48), "chunk_tokens"), (dict(n_table=1 << 27), "2^30"),
    (dict(head_dim=32), "head_dim"), (dict(n_kv=0), "head"), (dict(n_q=7), "head"), (dict(n_q=34), "head"), (dict(n_q=0), "head"),
    (dict(chunk_tokens=1 << 24), "slot"), (dict(n_seq=1 << 30, n_table=1 << 20), "too many"),
    (dict(n_seq=(1 << 31) - 1, n_table=1, n_q=2), "too many"),
    (dict(ws_bytes=0), "workspace"), (dict(ws_bytes=-1), "workspace"),
    (dict(q_ptr=P + 2), "16-byte"), (dict(slab_ptr=P + 8), "16-byte"), (dict(out_ptr=P + 4), "16-byte"), (dict(ws_ptr=P + 8), "16-byte"),
])
def test_attention_batch_refusals(bad, match):
    refused(mz.mz_attention_batch, **{**ATTENTION, **bad}, match=match)


def test_attention_batch_workspace():
    need = mz.mz_attention_batch_workspace_bytes(3, 8, 2, 64)
    assert need > 0
    refused(mz.mz_attention_batch, **{**ATTENTION, "ws_bytes": need - 1}, match="workspace")
    for bad in [(0, 8, 2, 64), (3, 7, 2, 64), (3, 8, 0, 64), (3, 8, 2, 32), (3, 0, 2, 64), (3, 34, 2, 64)]:
        assert mz.mz_attention_batch_workspace_bytes(*bad) == -1


@pytest.mark.parametrize("n_seq", [(1 << 31) - 1, 1 << 30, 1 << 24, 1 << 21])
def test_attention_batch_workspace_of_a_refused_batch(n_seq):
    assert mz.mz_attention_batch_workspace_bytes(n_seq, 8, 2, 64) == -1
    assert mz.mz_attention_batch_workspace_bytes(n_seq, (1 << 31) - 16, (1 << 31) - 16, 64) == -1
    refused(mz.mz_attention_batch, **{**ATTENTION, "n_seq": n_seq, "ws_bytes": 1 << 40}, match="too many")
    assert mz.mz_attention_batch_workspace_bytes((1 << 21) - 1, 8, 2, 64) > (1 << 21) * 4


LORA = dict(x_ptr=P, m=3, k=64, adapter_ptr=P, n_adapters=2, a_ptr=P, b_ptr=P, max_rank=16, n=100, base_ptr=P, y_ptr=P,
            y_stride=256, ws_ptr=P, ws_bytes=1 << 30)


@pytest.mark.parametrize("bad,match", [
    (dict(x_ptr=0), "NULL"), (dict(adapter_ptr=0), "NULL"), (dict(a_ptr=0), "NULL"), (dict(b_ptr=0), "NULL"),
    (dict(base_ptr=0), "NULL"), (dict(y_ptr=0), "NULL"), (dict(ws_ptr=0), "NULL"),
    (dict(m=-1), "positive"), (dict(n=0), "positive"), (dict(n_adapters=0), "n_adapters"), (dict(n_adapters=2048), "n_adapters"),
    (dict(k=0), "k must"), (dict(k=60), "k must"), (dict(k=-8), "k must"),
    (dict(max_rank=0), "max_rank"), (dict(max_rank=12), "max_rank"), (dict(max_rank=136), "max_rank"),
    (dict(y_stride=96), "y_stride"), (dict(y_stride=102), "y_stride"), (dict(y_stride=-4), "y_stride"),
    (dict(x_ptr=P + 2), "16-byte"), (dict(a_ptr=P + 8), "16-byte"), (dict(b_ptr=P + 8), "16-byte"),
    (dict(base_ptr=P + 4), "16-byte"), (dict(y_ptr=P + 4), "16-byte"), (dict(ws_ptr=P + 4), "16-byte"),
    (dict(m=1 << 30, n=1 << 30, y_stride=1 << 30), "too many"), (dict(n=1 << 30, y_stride=1 << 30), "too many"), (dict(ws_bytes=0), "workspace"), (dict(ws_bytes=-1), "workspace"),
])
def test_lora_add_refusals(bad, match):
    refused(mz.mz_lora_add, **{**LORA, **bad}, match=match)


def test_lora_workspace_and_no_rows():
    need = mz.mz_lora_workspace_bytes(3, 64, 16, 2)
    assert need > 0
    refused(mz.mz_lora_add, **{**LORA, "ws_bytes": need - 1}, match="workspace")
    for bad in [(0, 64, 16, 2), (3, 4, 16, 2), (3, 64, 4, 2), (3, 64, 129, 2), (3, 64, 16, 0), (3, 64, 16, 2048)]:
        assert mz.mz_lora_workspace_bytes(*bad) == -1
    # rows beyond those of one pass run as several in the same workspace
    most = max(mz.mz_lora_workspace_bytes(m, 4096, 64, 9) for m in range(1, 8193))
    for m in (8193, 9000, 1 << 20, (1 << 30) + 77):
        assert mz.mz_lora_workspace_bytes(8192, 4096, 64, 9) <= mz.mz_lora_workspace_bytes(m, 4096, 64, 9) <= most
    mz.mz_lora_add(**{**LORA, "m": 0, "ws_bytes": 0})


LOGITS = dict(logits_ptr=P, m=3, vocab=1000, stride=1024, out_ptr=P, token_ptr=P, ws_ptr=P, ws_bytes=1 << 20, penalty_ptr=P,
              history_ptr=P, history_off_ptr=P, bias_token_ptr=P, bias_value_ptr=P, bias_off_ptr=P, mask_ptr=P, n_masks=1,
              mask_words=32, mask_row_ptr=P)


@pytest.mark.parametrize("bad,match", [
    (dict(logits_ptr=0), "NULL"), (dict(out_ptr=0, token_ptr=0), "NULL"), (dict(logits_ptr=P + 2), "4-byte"),
    (dict(out_ptr=P + 1), "4-byte"), (dict(m=-1), "stride"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 30) + 1), "vocab"),
    (dict(stride=999), "stride"), (dict(stride=-1024), "stride"),
    (dict(history_off_ptr=0), "history"), (dict(penalty_ptr=0), "history"), (dict(bias_value_ptr=0), "bias"),
    (dict(bias_off_ptr=0), "bias"), (dict(mask_row_ptr=0), "mask"), (dict(n_masks=0), "mask"), (dict(mask_words=31), "mask"),
    (dict(m=(1 << 31) - 1, vocab=1 << 20, stride=1 << 20, mask_words=1 << 20), "too many"),
    (dict(ws_ptr=0), "workspace"), (dict(ws_bytes=0), "workspace"), (dict(ws_ptr=P + 2), "workspace"),
])
def test_logits_rules_refusals(bad, match):
    refused(mz.mz_logits_rules, **{**LOGITS, **bad}, match=match)


def test_logits_rules_workspace_and_no_rows():
    need = mz.mz_logits_rules_workspace_bytes(3, 1000)
    assert need > 0
    refused(mz.mz_logits_rules, **{**LOGITS, "ws_bytes": need - 1}, match="workspace")
    assert mz.mz_logits_rules_workspace_bytes(0, 1000) == -1 and mz.mz_logits_rules_workspace_bytes(3, 0) == -1
    mz.mz_logits_rules(**{**LOGITS, "m": 0, "ws_ptr": 0, "ws_bytes": 0})


def test_no_rows_of_empty_tensors():
    """An empty tensor's pointer is NULL."""
    mz.mz_kv_append(**{**APPEND, "m": 0, "k_ptr": 0, "v_ptr": 0, "q_ptr": 0, "q_out_ptr": 0, "seq_ptr": 0, "pos_ptr": 0})
    mz.mz_lora_add(**{**LORA, "m": 0, "x_ptr": 0, "adapter_ptr": 0, "base_ptr": 0, "y_ptr": 0, "ws_ptr": 0, "ws_bytes": 0})
    mz.mz_logits_rules(**{**LOGITS, "m": 0, "logits_ptr": 0, "out_ptr": 0, "token_ptr": 0, "ws_ptr": 0, "ws_bytes": 0})
    mz.mz_logits_rules(**{**LOGITS, "m": 0, "logits_ptr": 0, "out_ptr": 0, "penalty_ptr": 0, "mask_row_ptr": 0})
    # what is not rows is looked at all the same
    refused(mz.mz_logits_rules, **{**LOGITS, "m": 0, "history_off_ptr": 0}, match="history_off")
    refused(mz.mz_logits_rules, **{**LOGITS, "m": 0, "n_masks": 0}, match="mask")
    refused(mz.mz_kv_append, **{**APPEND, "m": 0, "slab_ptr": 0}, match="NULL")
    refused(mz.mz_lora_add, **{**LORA, "m": 0, "a_ptr": 0}, match="NULL")
    refused(mz.mz_lora_add, **{**LORA, "m": 0, "max_rank": 12}, match="max_rank")
    refused(mz.mz_logits_rules, **{**LOGITS, "m": 0, "stride": 999}, match="stride")


# ---- the largest calls and the workspaces of smaller ones: a launch holds fewer than 2^32 threads

def test_calls_beyond_one_launch():
    refused(mz.mz_attention_batch, **{**ATTENTION, "n_seq": 1 << 21, "ws_bytes": 1 << 40}, match="too many")      # 2^24 query rows
    refused(mz.mz_logits_rules, **{**LOGITS, "m": 1 << 23, "ws_bytes": 1 << 40}, match="too many")
    refused(mz.mz_logits_rules, **{**LOGITS, "m": 1 << 22, "vocab": 4097, "stride": 8192, "mask_words": 256, "ws_bytes": 1 << 40},
            match="too many")
    # a head of 32 alone: 4 items of 4 rows, 64-row tiles
    refused(mz.mz_kv_append, **{**APPEND, "n_q": 0, "n_kv": 1, "head_dim": 32, "m": 900 << 20}, match="too many")
    refused(mz.mz_lora_add, **{**LORA, "k": (1 << 30) + 8, "ws_bytes": 1 << 40}, match="k must")
    # 8 rows: a range of 256 columns each
    refused(mz.mz_lora_add, **{**LORA, "m": 8, "n": (1 << 29) + 1, "y_stride": (1 << 29) + 4, "ws_bytes": 1 << 40}, match="too many")
    for bad in [(3, 60, 16, 2), (3, (1 << 30) + 8, 16, 2), (3, 64, 12, 2)]:
        assert mz.mz_lora_workspace_bytes(*bad) == -1
    assert mz.mz_logits_rules_workspace_bytes(3, (1 << 30) + 1) == -1


@pytest.mark.parametrize("k,R,na", [(64, 8, 1), (2048, 16, 4), (4096, 64, 9), (8960, 128, 2047)])
def test_lora_workspace_of_the_largest_call_serves_all(k, R, na):
    need = [mz.mz_lora_workspace_bytes(m, k, R, na) for m in range(1, 8300)]
    assert need == sorted(need)


@pytest.mark.parametrize("vocab", [1, 1000, 4096, 4097, 128256, 151936, 1 << 21, 1 << 30])
def test_logits_workspace_of_the_largest_call_serves_all(vocab):
    need = [mz.mz_logits_rules_workspace_bytes(m, vocab) for m in range(1, 2000)]
    assert need == sorted(need) and need[0] >= 8


def test_attention_workspace_of_the_largest_call_serves_all():
    need = [mz.mz_attention_batch_workspace_bytes(b, 32, 8, 128) for b in range(1, 2000)]
    assert need == sorted(need)
