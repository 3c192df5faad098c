"""Sizes at which a launch would have 2^32 threads or more, which no dispatch holds: refused on the host. The
pointers are never read."""

import ctypes

import pytest

import paper_2609_02897_amd as asv
from paper_2609_02897_amd import _abi, _build

BIG = 1 << 50                  # between the fake arrays, so that none overlap


@pytest.fixture(scope="module")
def lib():
    if not _build.is_built():
        _build.build_library()
    return asv.load()


@pytest.mark.parametrize("type,ids", [(_abi.F32, 1024), (_abi.BF16, 2048), (_abi.F16, 2048)])
def test_adjust(lib, type, ids):
    for N, V in ((8 << 24, 1), ((8 << 24) - 7, ids), (8 << 23, ids + 1), (8 << 4, (1 << 30) - 1), (1 << 29, 3000)):
        if -(-N // 8) * -(-V // ids) < 1 << 24:
            continue
        a = _abi.AsvAdjustArgs()
        a.B, a.N, a.V, a.type = N, N, V, type
        a.in_, a.out, a.in_pitch, a.out_pitch = BIG, 3 * BIG, V, V
        assert lib.asv_adjust_logits(ctypes.byref(a), None) == asv.ASV_EINVAL, (N, V)


def test_counts(lib):
    for B, V in ((1 << 22, 1), (1 << 21, 20481), (1 << 29, 1000), (1 << 7, (1 << 30) - 1)):
        a = _abi.AsvCountsArgs()
        a.B, a.T, a.V, a.add = B, 9, V, 0
        a.tok, a.tok_offsets, a.counts, a.req_status = BIG, 2 * BIG, 3 * BIG, 9 * BIG
        assert lib.asv_token_counts(ctypes.byref(a), None) == asv.ASV_EINVAL, (B, V)


@pytest.mark.parametrize("layout", [0, 1, _abi.W_FP8])
def test_verify(lib, layout):
    def call(B, N, V, ruled):
        a = _abi.AsvVerifyArgs()
        a.B, a.N, a.H, a.V, a.w_lm_layout = B, N, 64, V, layout
        for i, f in enumerate(("hidden", "w_lm", "draft_tok", "parent", "req_offsets", "tau", "row_max",
                               "row_lse", "row_argmax", "drafted_logit", "accept", "accepted_len",
                               "bonus_token", "accepted_path", "req_status")):
            setattr(a, f, (i + 1) * BIG)
        a.params = asv.make_params()
        if ruled:
            rules = _abi.AsvLogitRules()
            rules.repetition = 90 * BIG
            return lib.asv_verify_ruled(ctypes.byref(a), ctypes.byref(rules), 80 * BIG, 1 << 60, None)
        if layout == _abi.W_FP8:
            return lib.asv_verify_ruled(ctypes.byref(a), None, 80 * BIG, 1 << 60, None)
        return lib.asv_verify(ctypes.byref(a), 80 * BIG, 1 << 60, None)

    # rows of the finishing step; workgroups of the LM head (256 ids x 256 rows at most)
    for B, N, V in ((1, (1 << 26) - 3, 5), (1 << 26, 1 << 26, 1), (3, 1 << 29, 256), (1, 1 << 20, 1 << 21)):
        assert call(B, N, V, False) == asv.ASV_EINVAL, (B, N, V)
    # with rules, whose rows are at most 65535
    V = 3 << 23                            # 98304 slabs x 256 row tiles of 256 rows, two launches at most
    if layout != _abi.W_FP8:
        assert call(1, 65535, V, True) == asv.ASV_EINVAL


def test_around_the_step(lib):
    B = 1 << 24
    status = lib.asv_draft_prune(BIG, B, None, 5, 2 * BIG, 3 * BIG, 4 * BIG, 5 * BIG, None)
    assert status == asv.ASV_EINVAL
    assert lib.asv_tree_meta(BIG, 2 * BIG, B, B, None, 0, 3 * BIG, None, 4 * BIG, None) == asv.ASV_EINVAL
    c = _abi.AsvCommitArgs()
    c.B = c.N = B
    for i, f in enumerate(("req_offsets", "draft_tok", "accepted_len", "accepted_path", "bonus_token",
                           "commit_off", "commit_tok", "commit_row", "req_status")):
        setattr(c, f, (i + 1) * BIG)
    assert lib.asv_commit(ctypes.byref(c), None) == asv.ASV_EINVAL


def test_draft_step(lib):
    d = _abi.AsvDraftArgs()
    d.B, d.H, d.V = 1 << 17, 64, 1 << 24         # 2^17 slabs x 2^11 row tiles of 128 ids x 256 rows
    for i, f in enumerate(("hidden", "w_draft", "tree", "topk_id", "topk_logp", "row_lse", "front_tok")):
        setattr(d, f, (i + 1) * BIG)
    d.shape = (ctypes.c_int32 * 3)(1, 1, 1)
    assert lib.asv_draft_step(ctypes.byref(d), 80 * BIG, 1 << 60, None) == asv.ASV_EINVAL
