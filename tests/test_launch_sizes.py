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
