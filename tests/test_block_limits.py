"""Largest sizes of the block cache calls, from their workspace queries: a call that no launch can hold is refused before anything
runs (a dimension of a grid has fewer than 2^32 threads), and its neighbours are not."""
import pytest

import block_cache_util as U
from paper_2506_19830_amd import binding as B

UNSUPPORTED = 2
UNITS = (1 << 22) + 64


def answer(fn, *args):
    try:
        return fn(*args)
    except B.LaError as e:
        assert e.status == UNSUPPORTED
        return None


@pytest.mark.parametrize("units,G,prefix,accepted", [
    (UNITS, 72, 40, False),                     # more than 64 rows to a group: workgroups of 1024
    ((1 << 22) - 1, 72, 40, True),
    (UNITS, 8, 40, True),                       # workgroups of 256
    (UNITS, 1, 2048 * 16, True),
    (UNITS, 1, 2048 * 16 + 1, False),           # more than 2048 blocks: 1024
    ((1 << 22) - 1, 1, 2048 * 16 + 1, True),
    (1 << 23, 1, 40, True),
    ((1 << 23) + 1, 1, 40, False),
])
def test_select(units, G, prefix, accepted):
    d = U.desc("bf16", Hq=G, Hkv=1, gamma=units, bs=16, max_blocks=4096)
    got = answer(B.la_block_select_workspace, d, B.make_select_desc(group_len=1, max_blocks=1), [prefix])
    assert (got is not None) == accepted
    if accepted:
        assert got >= units * -(-prefix // 16) * 12


@pytest.mark.parametrize("rows,prefix,accepted", [
    ((1 << 28) - 64, 20000, True),              # two workgroups to a unit: 16 threads a row join them
    ((1 << 28) + (1 << 20), 20000, False),
    ((1 << 28) + (1 << 20), 1000, True),        # one: nothing to join
])
def test_attention_whose_keys_are_split(rows, prefix, accepted):
    d = U.desc("bf16", Hq=1, Hkv=1, D=64, gamma=rows, bs=16, max_blocks=2048)
    got = answer(B.la_verify_attention_sparse_workspace, d, None, [prefix])
    assert (got is not None) == accepted
    if accepted:
        assert got == 0 if prefix == 1000 else got >= 2 * rows * 66 * 4


def test_attention_over_lists():
    """A unit per row: 2^23 workgroups of four wavefronts can be launched, of eight not."""
    s = B.make_select_desc(group_len=1, max_blocks=1)
    for units, accepted in (((1 << 23) - 8, True), (1 << 23, True), ((1 << 23) + 8, False)):
        d = U.desc("mxfp4_e2m1", Hq=8, Hkv=8, D=64, gamma=units // 8, bs=16, max_blocks=1)
        assert (answer(B.la_verify_attention_sparse_workspace, d, s, [16]) is not None) == accepted


def test_forced_shapes():
    """The self-test hook: shapes that a head dimension does not have are refused, and the choice comes back."""
    B.select_library("bench")
    try:
        s = B.make_select_desc(group_len=1, max_blocks=4)
        want = {D: B.la_verify_attention_sparse_workspace(U.desc("bf16", D=D), s, [100]) for D in (64, 256)}
        for D, shape, exists in ((64, (16, 4), True), (64, (128, 8), True), (64, (128, 4), False), (64, (48, 4), False),
                                 (256, (128, 4), True), (256, (16, 8), False), (256, (64, 4), False)):
            B.la_selftest_sparse_plan(*shape, 2)
            got = answer(B.la_verify_attention_sparse_workspace, U.desc("bf16", D=D), s, [100])
            assert got is None if not exists else got >= 2 * 4 * (D + 2) * 4
        with pytest.raises(B.LaError):
            B.la_selftest_sparse_plan(-1, 4, 1)
        B.la_selftest_sparse_plan()
        assert want == {D: B.la_verify_attention_sparse_workspace(U.desc("bf16", D=D), s, [100]) for D in (64, 256)}
    finally:
        B.la_selftest_sparse_plan()
        B.select_library("product")
