"""Where adjust_logits may write: the input itself, or rows that share no element with it, in the same buffer too."""

import ctypes

import numpy as np
import pytest

import paper_2609_02897_amd as asv
from paper_2609_02897_amd import _abi, _build

BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not _build.is_built():
        _build.build_library()
    return asv.load()


def test_shared_elements_are_refused(lib):
    """On the host; the pointers are never read."""
    def call(shift, in_pitch, out_pitch, N=9, V=300, type=_abi.F32):
        a = _abi.AsvAdjustArgs()
        a.B, a.N, a.V, a.type = N, N, V, type
        a.in_, a.out, a.in_pitch, a.out_pitch = BIG, BIG + shift, in_pitch, out_pitch
        return lib.asv_adjust_logits(ctypes.byref(a), None)

    for shift, p, q in ((4, 300, 300), (-4, 300, 300), (1200, 300, 300), (1200, 599, 599), (1196, 600, 600),
                        (1204, 600, 600), (-1204, 600, 600), (4 * 899, 600, 600), (4 * 901, 600, 600),
                        (1196, 1000, 1000), (4 * 701, 1000, 1000),
                        (1200, 600, 601), (1200, 601, 600), (0, 300, 304)):
        assert call(shift, p, q) == asv.ASV_EINVAL, (shift, p, q)
    for shift, p in ((598, 600), (602, 600), (2, 300)):
        assert call(shift, p, p, type=_abi.BF16) == asv.ASV_EINVAL, (shift, p)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("N,V,pitch,shift", [(9, 300, 600, 300), (9, 300, 1000, 300), (9, 300, 1000, 700),
                                             (5, 33, 100, 45), (1, 300, 300, 300), (70, 256, 512, 256)])
def test_rows_between_each_other(dtype, N, V, pitch, shift):
    """Both halves of one buffer's rows, in either order; what lies between stays."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev, dt = torch.device("cuda:0"), getattr(torch, dtype)
    g = torch.Generator(device=dev).manual_seed(V)
    rules = asv.LogitRules(bias=torch.randn(V, device=dev, generator=g))
    x = torch.randn((N, V), device=dev, generator=g).to(dt)
    want = asv.adjust_logits(x, rules)
    for a, b in ((0, shift), (shift, 0)):
        buf = torch.full((N + 1, pitch), 7.0, dtype=dt, device=dev).view(-1)
        views = [buf[k:k + N * pitch].view(N, pitch)[:, :V] for k in (a, b)]
        views[0].copy_(x)
        assert asv.adjust_logits(views[0], rules, out=views[1]) is views[1]
        assert torch.equal(views[0], x) and torch.equal(views[1], want)
        for v in views:
            v.fill_(7.0)
        assert bool((buf == 7.0).all())


@pytest.mark.gpu
def test_one_row_in_place_under_two_strides():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    V, dev = 300, torch.device("cuda:0")
    buf = torch.randn((4, 512), device=dev)
    rules = asv.LogitRules(bias=torch.from_numpy(np.arange(V, dtype=np.float32)).to(dev))
    want = asv.adjust_logits(buf[2:3, :V], rules)
    same = buf.view(-1)[1024:1024 + V].view(1, V)
    asv.adjust_logits(buf[2:3, :V], rules, out=same)
    assert torch.equal(same, want)
