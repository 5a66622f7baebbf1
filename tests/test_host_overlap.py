"""Arrays of a step's tables that overlap: refused before anything is launched. The addresses are
never used, since every call is refused."""

import ctypes as C

import pytest

import paper_2512_04013_amd as aug

READ = dict(ctx_len=16, q_len=16, parents=32)                   # bytes of 4 requests and 8 rows
WRITTEN = dict(block_table=64, held=16, free_ids=64, free_count=4, q_start=20, kv_len=16, state=16, positions=32, slots=64, seen=64,
               scratch=16)


def _args(**kw):
    f = dict(num_reqs=4, max_rows=8, max_blocks=4, num_pool_blocks=16, max_draft=4, reserved=0)
    f.update({name: (i + 1) << 20 for i, name in enumerate([*READ, *WRITTEN])})
    f.update(kw)
    return aug.aug_step_tables_args(**f)


@pytest.mark.parametrize("read", READ)
@pytest.mark.parametrize("written", WRITTEN)
def test_read_over_written(read, written):
    base = _args()
    at = getattr(base, written)
    for offset in {0, min(4, WRITTEN[written] - 4), WRITTEN[written] - 4, 4 - READ[read]}:
        if offset == 0 and (read, written) == ("ctx_len", "kv_len"):
            continue                                            # the one that is allowed
        a = _args(**{read: at + offset})
        assert aug.lib().aug_step_tables(C.byref(a), None) == aug.AUG_ERR_INVALID, offset
        assert f"{read} overlaps {written}" in aug.aug_last_error()


def test_rows_count_as_lengths_do():
    """q_len is not kv_len, also where ctx_len is."""
    a = _args()
    a = _args(ctx_len=a.kv_len, q_len=a.kv_len)
    assert aug.lib().aug_step_tables(C.byref(a), None) == aug.AUG_ERR_INVALID and "q_len overlaps kv_len" in aug.aug_last_error()
