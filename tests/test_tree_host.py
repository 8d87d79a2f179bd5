"""Refusals of the calls that check drafted trees: every one is found on the
host before anything is enqueued, so they need no GPU.  The device pointers are
never followed."""

import ctypes
import glob
import os
import re

import pytest

from paper_2609_01338_amd import mz
from test_batch_host import APPEND, refused

P = 1 << 20          # stands for device pointers on 16-byte boundaries, far apart


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(mz.LIB_PATH):
        from paper_2609_01338_amd import build
        build.build_all()
    mz.lib()


PLAN = dict(row_off_ptr=P, lens_ptr=2 * P, n_seq=3, m=9, parent_ptr=3 * P, seq_ptr=4 * P, place_ptr=5 * P, rope_pos_ptr=6 * P,
            mask_ptr=7 * P, mask_words=2)


@pytest.mark.parametrize("bad,match", [
    (dict(row_off_ptr=0), "NULL"), (dict(lens_ptr=0), "NULL"),
    (dict(n_seq=0), "n_seq"), (dict(n_seq=(1 << 20) + 1), "n_seq"), (dict(m=-1), "m must"), (dict(m=(1 << 30) + 1), "m must"),
    (dict(seq_ptr=0, place_ptr=0, rope_pos_ptr=0, mask_ptr=0, mask_words=0), "no output"),
    (dict(mask_words=0), "mask_words"), (dict(mask_words=33), "mask_words"), (dict(mask_words=-1), "mask_words"),
    (dict(mask_ptr=0), "without a mask"),
    (dict(seq_ptr=5 * P + 32), "overlap"), (dict(mask_ptr=6 * P - 71), "overlap"), (dict(place_ptr=2 * P + 8), "overlap"),
    (dict(rope_pos_ptr=3 * P - 4), "overlap"), (dict(seq_ptr=P - 35), "overlap"),
])
def test_plan_refusals(bad, match):
    refused(mz.mz_tree_plan, **{**PLAN, **bad}, match=match)


def test_plan_no_rows():
    mz.mz_tree_plan(**{**PLAN, "m": 0})
    mz.mz_tree_plan(P, P, 1, 0)


AXES = {**APPEND, "rope_pos_ptr": P, "n_axes": 2, "pair_axis": [0, 1] * 16}


@pytest.mark.parametrize("bad,match", [
    (dict(n_axes=0), "n_axes"), (dict(n_axes=5), "n_axes"), (dict(rope_pos_ptr=0), "NULL"), (dict(pair_axis=None), "NULL"),
    (dict(pair_axis=[0] * 31 + [2]), "axis 2 of 2"), (dict(pair_axis=[254] + [0] * 31), "axis 254 of 2"), (dict(n_axes=1), "axis 1 of 1"),
    (dict(pair_axis=[0] * 31), "pairs"), (dict(pair_axis=[0] * 33), "pairs"),
    (dict(m=-1), "negative"), (dict(k_ptr=0), "NULL"), (dict(seq_ptr=0), "NULL"), (dict(slab_ptr=0), "NULL"), (dict(n_rope=0), "n_rope"),
    (dict(n_kv=0), "head"), (dict(chunk_tokens=24), "chunk_tokens"), (dict(k_stride=124), "stride"), (dict(k_ptr=P + 4), "16-byte"),
    (dict(n_table=1 << 27), "2^30"), (dict(m=(1 << 31) - 1, n_q=1024, n_kv=1024, head_dim=128, pair_axis=[0] * 64), "too many"),
])
def test_append_axes_refusals(bad, match):
    refused(mz.mz_kv_append_axes, **{**AXES, **bad}, match=match)


def test_append_axes_null_structs_and_no_rows():
    mz.mz_kv_append_axes(**{**AXES, "m": 0, "k_ptr": 0, "v_ptr": 0, "q_ptr": 0, "q_out_ptr": 0, "seq_ptr": 0, "pos_ptr": 0, "rope_pos_ptr": 0})
    lib = mz.lib()
    assert lib.mz_kv_append_axes(None, None, 0, None) == mz.MZ_EINVAL
    a = mz.mz_kv_append_args(0, P, P, 0, 0, 0, 1, 64, 0, 1, P, P, P, 4, 4, P, P, 1, 1, 16, 0)
    assert lib.mz_kv_append_axes(ctypes.byref(a), None, 0, None) == mz.MZ_EINVAL


ATTENTION = dict(q_ptr=P, m=9, row_off_ptr=P, lens_ptr=P, n_seq=3, slab_ptr=P, n_slots=8, table_ptr=P, n_table=4, chunk_tokens=16,
                 n_q=8, n_kv=2, head_dim=64, ws_ptr=P, ws_bytes=1 << 40, out_ptr=P, mask_ptr=P, mask_words=1)


@pytest.mark.parametrize("bad,match", [
    (dict(q_ptr=0), "NULL"), (dict(row_off_ptr=0), "NULL"), (dict(lens_ptr=0), "NULL"), (dict(slab_ptr=0), "NULL"),
    (dict(table_ptr=0), "NULL"), (dict(ws_ptr=0), "NULL"), (dict(out_ptr=0), "NULL"),
    (dict(m=-1), "negative"), (dict(n_seq=0), "positive"), (dict(n_seq=(1 << 20) + 1), "n_seq"), (dict(n_slots=0), "positive"),
    (dict(n_table=0), "positive"), (dict(n_table=1 << 27), "2^30"), (dict(chunk_tokens=4), "chunk_tokens"), (dict(chunk_tokens=24), "chunk_tokens"),
    (dict(mask_words=0), "mask_words"), (dict(mask_words=33), "mask_words"), (dict(mask_words=-1), "mask_words"), (dict(mask_ptr=0), "without a mask"),
    (dict(head_dim=32), "head_dim"), (dict(head_dim=96), "head_dim"), (dict(n_kv=0), "head"), (dict(n_q=9), "head"), (dict(n_q=1), "head"),
    (dict(n_q=34, n_kv=2), "head"), (dict(m=1 << 21), "too many"), (dict(m=0, n_q=1 << 25, n_kv=1 << 24), "too many"),
    (dict(chunk_tokens=1 << 23, n_table=1), "slot"), (dict(n_seq=1 << 20, m=1000, n_table=1 << 20), "too many"),
    (dict(q_ptr=P + 8), "16-byte"), (dict(slab_ptr=P + 8), "16-byte"), (dict(out_ptr=P + 2), "16-byte"), (dict(ws_ptr=P + 4), "16-byte"),
])
def test_attention_tree_refusals(bad, match):
    refused(mz.mz_attention_tree, **{**ATTENTION, **bad}, match=match)


APART = {**ATTENTION, "q_ptr": 2 * P, "row_off_ptr": 3 * P, "lens_ptr": 4 * P, "slab_ptr": 100 * P, "table_ptr": 5 * P, "mask_ptr": 6 * P,
         "out_ptr": 7 * P, "ws_ptr": 2000 * P}


@pytest.mark.parametrize("bad,match", [
    (dict(out_ptr=2 * P + 64), "overlaps an input"), (dict(out_ptr=4 * P), "overlaps an input"), (dict(out_ptr=6 * P), "overlaps an input"),
    (dict(out_ptr=100 * P + 1024), "overlaps an input"), (dict(table_ptr=2004 * P), "overlaps an input"), (dict(ws_ptr=100 * P), "overlaps an input"),
    (dict(ws_ptr=7 * P), "two outputs"), (dict(out_ptr=2000 * P + 256), "two outputs"),
])
def test_attention_tree_outputs_that_overlap(bad, match):
    refused(mz.mz_attention_tree, **{**APART, **bad}, match=match)


@pytest.mark.parametrize("bad,match", [(dict(n_layers=4097), "at most 4096"), (dict(layer_bytes=(1 << 48) + 16), "2^48")])
def test_layers_that_are_too_many_or_far(bad, match):
    refused(mz.mz_tree_accept, **{**ACCEPT, **bad}, match=match)
    refused(mz.mz_kv_copy, **{**COPY, **bad}, match=match)


def test_attention_tree_workspace():
    need = mz.mz_attention_tree_workspace_bytes(9, 3, 8, 2, 64)
    assert need > 0
    refused(mz.mz_attention_tree, **{**ATTENTION, "ws_bytes": need - 1}, match="workspace")
    for bad in ((0, 3, 8, 2, 64), (9, 0, 8, 2, 64), (9, 3, 8, 0, 64), (9, 3, 9, 2, 64), (9, 3, 34, 2, 64), (9, 3, 8, 2, 32),
                (1 << 21, 3, 8, 2, 64), (9, (1 << 20) + 1, 8, 2, 64), (9, 3, -8, -2, 64)):
        assert mz.mz_attention_tree_workspace_bytes(*bad) == -1
    for nq, nkv, hd in ((8, 2, 64), (32, 8, 128), (16, 1, 64)):      # one for the most rows and sequences serves fewer
        sizes = [[mz.mz_attention_tree_workspace_bytes(m, n, nq, nkv, hd) for n in (1, 2, 3, 7, 64, 300, 5000)] for m in (1, 2, 5, 16, 33, 200, 4000)]
        for row in sizes:
            assert row == sorted(row)
        for column in zip(*sizes):
            assert list(column) == sorted(column)


def test_attention_tree_no_rows():
    mz.mz_attention_tree(**{**ATTENTION, "m": 0, "q_ptr": 0, "out_ptr": 0, "mask_ptr": 0, "ws_ptr": 0, "ws_bytes": 0})


ACCEPT = dict(row_off_ptr=P, token_ptr=2 * P, choice_ptr=3 * P, lens_ptr=4 * P, n_seq=3, m=9, accepted_ptr=5 * P, path_ptr=6 * P,
              next_ptr=7 * P, len_out_ptr=8 * P, parent_ptr=9 * P, slab_ptr=100 * P, n_slots=8, n_layers=2, layer_bytes=65536,
              table_ptr=10 * P, n_table=4, chunk_tokens=16, n_kv=2, head_dim=64)


@pytest.mark.parametrize("bad,match", [
    *[({k + "_ptr": 0}, "NULL") for k in ("row_off", "token", "choice", "lens", "accepted", "path", "next", "len_out", "slab", "table")],
    (dict(n_seq=0), "n_seq"), (dict(n_seq=(1 << 20) + 1), "n_seq"), (dict(m=-1), "m must"), (dict(m=(1 << 30) + 1), "m must"),
    (dict(n_layers=-1), "n_layers"), (dict(n_slots=0), "positive"), (dict(n_table=0), "positive"), (dict(chunk_tokens=12), "chunk_tokens"),
    (dict(n_table=1 << 27), "2^30"), (dict(head_dim=48), "head_dim"), (dict(n_kv=0), "head"), (dict(n_kv=1025), "head"),
    (dict(layer_bytes=65535 * 8), "16-byte"), (dict(layer_bytes=65520), "layers overlap"), (dict(layer_bytes=0), "layers overlap"),
    (dict(slab_ptr=100 * P + 8), "16-byte"), (dict(chunk_tokens=1 << 22, n_table=1), "slot"),
    (dict(len_out_ptr=4 * P), "overlaps an input"), (dict(path_ptr=2 * P), "overlaps an input"), (dict(next_ptr=5 * P + 8), "two outputs"),
    (dict(slab_ptr=10 * P - 16), "overlap"), (dict(n_seq=1 << 20, n_kv=16, head_dim=128, layer_bytes=1 << 30), "too many"),
])
def test_accept_refusals(bad, match):
    refused(mz.mz_tree_accept, **{**ACCEPT, **bad}, match=match)


PAGES = dict(table_ptr=P, table_out_ptr=2 * P, n_seq=3, n_table=5, n_slots=40, chunk_tokens=16, keep_ptr=3 * P, copies_ptr=4 * P, info_ptr=5 * P,
             ws_ptr=6 * P, ws_bytes=1 << 19, src_ptr=7 * P, room_ptr=8 * P)


@pytest.mark.parametrize("bad,match", [
    *[({k + "_ptr": 0}, "NULL") for k in ("table", "table_out", "keep", "copies", "info", "ws")],
    (dict(n_seq=0), "positive"), (dict(n_table=0), "positive"), (dict(n_slots=0), "positive"), (dict(chunk_tokens=20), "chunk_tokens"),
    (dict(n_table=1 << 27), "2^30"), (dict(n_seq=(1 << 20) + 1), "too many"), (dict(n_seq=1 << 15, n_table=1 << 14), "too many"),
    (dict(n_slots=(1 << 28) + 1), "too many"), (dict(slot_limit=-1), "slot_limit"), (dict(slot_limit=41), "slot_limit"),
    (dict(copies_ptr=4 * P + 8), "16-byte"), (dict(ws_ptr=6 * P + 4), "16-byte"),
    (dict(table_out_ptr=P + 4), "overlaps an input"), (dict(table_out_ptr=3 * P), "overlaps an input"), (dict(copies_ptr=P), "overlaps an input"),
    (dict(info_ptr=7 * P), "overlaps an input"), (dict(info_ptr=6 * P + 256), "two outputs"), (dict(copies_ptr=2 * P), "two outputs"),
])
def test_pages_refusals(bad, match):
    refused(mz.mz_kv_pages, **{**PAGES, **bad}, match=match)


def test_pages_workspace():
    need = mz.mz_kv_pages_workspace_bytes(3, 5, 40)
    refused(mz.mz_kv_pages, **{**PAGES, "ws_bytes": need - 1}, match="workspace")
    for bad in ((0, 5, 40), (3, 0, 40), (3, 5, 0), ((1 << 20) + 1, 1, 1), (1 << 15, 1 << 14, 4), (3, 5, (1 << 28) + 1)):
        assert mz.mz_kv_pages_workspace_bytes(*bad) == -1
    sizes = [mz.mz_kv_pages_workspace_bytes(a, b, c) for a, b, c in ((1, 1, 1), (1, 9, 1), (5, 9, 1), (5, 9, 700), (64, 9, 700), (64, 900, 70000))]
    assert sizes == sorted(sizes)


COPY = dict(copies_ptr=P, n_copies_ptr=P, max_copies=4, slab_ptr=P, n_slots=8, n_layers=2, layer_bytes=131072, chunk_tokens=16, n_kv=2, head_dim=64)


@pytest.mark.parametrize("bad,match", [
    (dict(copies_ptr=0), "NULL"), (dict(n_copies_ptr=0), "NULL"), (dict(slab_ptr=0), "NULL"), (dict(max_copies=-1), "max_copies"),
    (dict(n_layers=0), "n_layers"), (dict(n_slots=0), "positive"), (dict(chunk_tokens=4), "chunk_tokens"), (dict(head_dim=16), "head_dim"),
    (dict(n_kv=0), "head"), (dict(copies_ptr=P + 4), "16-byte"), (dict(slab_ptr=P + 4), "16-byte"), (dict(layer_bytes=131080), "16-byte"),
    (dict(layer_bytes=65536 - 16), "layers overlap"), (dict(layer_bytes=-131072), "layers overlap"), (dict(chunk_tokens=1 << 22), "slot"),
])
def test_copy_refusals(bad, match):
    refused(mz.mz_kv_copy, **{**COPY, **bad}, match=match)


def test_copy_of_nothing():
    mz.mz_kv_copy(**{**COPY, "max_copies": 0, "copies_ptr": 0, "n_copies_ptr": 0})


def test_assembly_that_writes_m0_says_so():
    """The compiler may hold a value of its own in M0 across a block that does not name it."""
    seen = 0
    for path in glob.glob(os.path.join(os.path.dirname(mz.__file__), "csrc", "*")):
        with open(path) as f:
            text = f.read()
        for block in re.findall(r"\basm\b(?:\s+volatile)?\s*\(.*?\)\s*;", text, re.S):
            if re.search(r"\bm0\s*,", block.split("::")[0]):
                seen += 1
                assert '"m0"' in block, (os.path.basename(path), block)
    assert seen >= 6
