"""Queries and outputs of tree attention that overlap in part: refused before anything is launched. The addresses are
never used."""

import ctypes as C

import pytest

import paper_2512_04013_amd as aug

P = 1 << 20


@pytest.mark.parametrize("kv,size", [("bf16", 2), ("f32", 4)])
def test_partial_overlap(kv, size):
    io = "f32" if kv == "f32" else "bf16"
    shape = aug.make_shape(8, 2, 128, io, kv, io, 0.1)
    batch = aug.aug_tree_batch(num_reqs=4, max_rows=32, max_blocks=17, max_draft=8, q_start=P, kv_len=P, block_table=P, seen=P)
    whole = 32 * 8 * 128 * size
    for offset in (16, -16, 8 * 128 * size, whole - 16, 16 - whole):
        status = aug.lib().aug_attn_tree(C.byref(shape), C.byref(batch), P, 1 << 30, P, P, P, P, 4, (1 << 30) + offset, P, 1 << 40, None)
        assert status == aug.AUG_ERR_INVALID and "overlap" in aug.aug_last_error(), offset
