"""The 8-bit LM head against float64: its quantisation code for code, the logits of lm_head_logits, and
verification on it. Tolerance of a logit: the products of two codes are exact in fp32 (8 significant
bits), their scales are powers of two, and a logit is the fp32 sum of H products, each of whose H - 1 additions
is off by at most 2^-24 of a partial sum, itself at most S = sum |x w|: (H - 1) 2^-24 S. Stored in 16 bits, half a step
more: 2^-8 (bf16) or 2^-11 (fp16) of the logit, and half of fp16's smallest step, 2^-25."""

import numpy as np
import pytest

import oracle
import rules_oracle as ro
from harness import compare, to_host
from workloads import bf16_normal, bf16_weights, build_tree, custom_workload

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def asv():
    import paper_2609_02897_amd as m
    m.load()
    return m


def _bf16(bits, dev):
    import torch
    return torch.from_numpy(np.array(bits, dtype=np.uint16).view(np.int16)).to(dev).view(
        torch.bfloat16)


def _to_bits(x):
    """bf16 bits of values that bf16 holds exactly."""
    return (np.asarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def _case(N, V, H, seed=0):
    rng = np.random.default_rng([seed, N, V, H])
    x, w = bf16_normal(rng, (N, H), 1.0), bf16_normal(rng, (V, H), 0.05)
    # blocks of other magnitudes, zeros among them
    xf = oracle.widen_bf16(x) * 2.0 ** rng.integers(-9, 9, (N, 1))
    xf[:, :64] *= rng.random((N, 1)) < 0.7
    wf = oracle.widen_bf16(w) * 2.0 ** rng.integers(-3, 4, (V, 1))
    return _to_bits(xf), _to_bits(wf)


def _check_logits(got, xq, wq, dtype):
    H = xq.shape[1]
    z, S = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
    tol = (H - 1) * 2.0 ** -24 * S + {"float32": 0 * z, "bfloat16": 2.0 ** -8 * np.abs(z),
                                      "float16": 2.0 ** -11 * np.abs(z) + 2.0 ** -25}[dtype]
    bad = np.argwhere(~(np.abs(got - z) <= tol))
    assert len(bad) == 0, (bad[:4], got[tuple(bad[0])], z[tuple(bad[0])])


SHAPES = [(1, 1, 64), (1, 257, 128), (3, 5, 64), (16, 127, 192), (17, 128, 576), (60, 1000, 320),
          (64, 255, 4096), (65, 256, 128), (128, 513, 192), (129, 300, 256), (193, 1025, 64),
          (257, 129, 448), (300, 700, 320), (2, 33, 4160), (5, 260, 8320), (130, 270, 8256),
          # every cut of the ids: 64-, 128- and 256-id tiles, tails of 64 and 128 ids behind rounds
          (7, 20001, 64), (60, 40003, 64), (64, 50001, 64), (33, 70001, 64), (9, 90001, 64),
          (3, 140001, 64), (4, 152001, 64), (5, 168003, 64), (6, 180003, 64), (2, 200001, 64),
          (100, 32000, 64), (90, 75003, 64), (190, 20000, 64), (333, 40003, 128), (150, 36003, 64),
          (500, 18000, 64), (230, 67003, 64), (190, 16003, 64), (200, 14001, 64)]


@pytest.mark.parametrize("N,V,H", SHAPES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_logits(asv, dev, N, V, H, dtype):
    import torch
    x, w = _case(N, V, H)
    head = asv.quantize_lm_head(_bf16(w, dev))
    got = asv.lm_head_logits(_bf16(x, dev), head, dtype=getattr(torch, dtype))
    assert got.shape == (N, V) and got.dtype == getattr(torch, dtype)
    _, _, xq = ro.quantise(oracle.widen_bf16(x), 1)
    _, _, wq = ro.quantise(oracle.widen_bf16(w), 128)
    _check_logits(got.double().cpu().numpy(), xq, wq, dtype)


@pytest.mark.parametrize("V,H", [(1, 64), (128, 128), (129, 192), (300, 320), (513, 4160)])
def test_packed_copy(asv, dev, V, H):
    """quantize_lm_head, pack_lm_head_fp8 of the same codes and the layout of asv.h, byte for byte."""
    import torch
    _, w = _case(1, V, H)
    codes, scale, _ = ro.quantise(oracle.widen_bf16(w), 128)
    S, K = -(-V // 256), -(-H // 128)
    P = -(-K // 4) * 4
    pad = np.zeros((S * 256, H), dtype=np.uint8)
    pad[:V] = codes
    want = pad.reshape(S, 256, H // 64, 2, 4, 8).transpose(2, 0, 1, 4, 3, 5).ravel()
    a = asv.quantize_lm_head(_bf16(w, dev))
    b = asv.pack_lm_head_fp8(torch.from_numpy(codes).to(dev).view(torch.float8_e4m3fn),
                             torch.from_numpy(scale).to(dev).view(torch.float8_e8m0fnu))
    for head in (a, b):
        data = head.data.cpu().numpy()
        assert len(data) == S * 256 * H + 2 * S * P
        got, sc = data[:want.size], data[want.size:].reshape(2 * S, P)[:scale.shape[0], :K]
        # a zero's sign is free
        assert np.array_equal(np.where(got == 128, 0, got), np.where(want == 128, 0, want))
        assert np.array_equal(sc, scale)


def test_every_bf16_value_is_rounded_to_the_nearest_code(asv, dev):
    """Through an identity weight: every finite bf16 value, in blocks whose largest is 2^e."""
    import torch
    H = 128
    w = np.zeros((H, H))
    np.fill_diagonal(w, 1.0)
    head = asv.quantize_lm_head(_bf16(_to_bits(w), dev))
    bits = np.arange(0x7f80, dtype=np.uint16)
    vals = np.concatenate([bits, bits | 0x8000])
    rows = []
    for top in (0x0001, 0x0080, 0x3f80, 0x3fe0, 0x3fe1, 0x4000, 0x43e0, 0x7e80):   # each block's largest
        mine = vals[(vals & 0x7fff) <= top][-127 * 400:]
        mine = np.concatenate([mine, np.zeros(-len(mine) % 127, dtype=np.uint16)]).reshape(-1, 127)
        rows.append(np.concatenate([mine, np.full((len(mine), 1), top, dtype=np.uint16)], 1))
    x = np.concatenate(rows)
    got = asv.lm_head_logits(_bf16(x, dev), head).cpu().numpy().astype(np.float64)
    _, _, want = ro.quantise(oracle.widen_bf16(x), 1)
    # fp32 holds every product exactly, except below its smallest normal number, where it may be flushed
    small = np.abs(want) < 2.0 ** -126
    assert np.array_equal(got[~small], want[~small])
    assert np.all(np.abs(got[small]) < 2.0 ** -126)


def test_infinities_and_nans_stay_in_their_rows_and_blocks(asv, dev):
    N, V, H = 20, 300, 384
    x, w = _case(N, V, H, 3)
    x[3, 5], x[7, 383], w[200, 130] = 0x7f80, 0x7fc0, 0xff80      # inf, NaN; -inf: ids 128 .. 255
    got = asv.lm_head_logits(_bf16(x, dev), asv.quantize_lm_head(_bf16(w, dev))).cpu().numpy()
    bad = np.zeros((N, V), dtype=bool)
    bad[[3, 7]] = True
    bad[:, 128:256] = True
    assert np.array_equal(np.isnan(got), bad)


@pytest.mark.parametrize("pitch", [300, 304, 307, 512])
def test_rows_apart_and_what_lies_between_them(asv, dev, pitch):
    import torch
    N, V, H = 70, 300, 192
    x, w = _case(N, V, H, 4)
    head = asv.quantize_lm_head(_bf16(w, dev))
    for dtype in (torch.float32, torch.bfloat16):
        whole = asv.lm_head_logits(_bf16(x, dev), head, dtype=dtype)
        for first in (0, 1):
            buf = torch.full((N + 2, pitch + 1), 7.0, dtype=dtype, device=dev)
            out = buf.view(-1)[first:first + (N + 1) * pitch].view(N + 1, pitch)[:N, :V]
            assert asv.lm_head_logits(_bf16(x, dev), head, out=out) is out
            assert torch.equal(out, whole)
            out.fill_(7.0)
            assert bool((buf == 7.0).all())


@pytest.mark.parametrize("kind,n_req,H,V", [("tiny", 1, 64, 300), ("eagle60", 1, 320, 3001),
                                            ("adaptive", 3, 192, 2500), ("level8x8", 5, 128, 1300)])
def test_verify(asv, dev, kind, n_req, H, V):
    """Verification on the 8-bit head is verification on the values that its codes stand for, policy
    and draft confidence included."""
    rng = np.random.default_rng([n_req, H, V])
    trees = [build_tree(kind, rng, b) for b in range(n_req)]
    w = custom_workload("fp8", H, V, trees, 0.2, seed=5, w_std=0.09, draft_logits=True)
    W = bf16_weights(V, H, 0.09, 77)
    _, _, xq = ro.quantise(oracle.widen_bf16(w.hidden), 1)
    _, _, wq = ro.quantise(oracle.widen_bf16(W), 128)
    w.with_drafts(oracle.row_top8(xq @ wq.T))
    st = [oracle.state_init(oracle.Params()) for _ in range(w.B)]
    ref = oracle.verify(wq, _to_bits(xq), w.draft_tok, w.parent, w.req_offsets, w.tau,
                        w.draft_logits, st)
    import torch
    t = lambda a: torch.from_numpy(np.array(a, order="C")).to(dev)   # noqa: E731
    state = asv.state_init(w.B, device=dev)
    head = asv.quantize_lm_head(_bf16(W, dev))
    args = (_bf16(w.hidden, dev), head, t(w.draft_tok.astype(np.int32)),
            t(w.parent.astype(np.int32)), t(w.req_offsets.astype(np.int32)), t(w.tau),
            t(w.draft_logits))
    out = asv.verify(*args, state=state)
    got = to_host(out)
    compare(w, ref, got)
    from harness import compare_state
    banded = set(np.flatnonzero(ref["band_at"] >= 0))
    compare_state(asv.state_fields(state), ref["state"], banded_requests=banded)
    # the logits' own operator agrees with the records
    z = asv.lm_head_logits(args[0], head)
    assert torch.equal(z.max(1).values, out.row_max)


def test_verify_workspace_of_a_larger_batch(asv, dev):
    import torch
    H, V = 192, 900
    W = bf16_weights(V, H, 0.09, 8)
    head = asv.quantize_lm_head(_bf16(W, dev))
    ws = asv.alloc_workspace(9, 300, H, V, dev, head)
    for B, n in ((1, 5), (9, 33)):
        N = B * n
        x = _bf16(bf16_normal(np.random.default_rng([B, n]), (N, H), 1.0), dev)
        par = torch.arange(N, dtype=torch.int32, device=dev) - 1
        off = torch.arange(0, N + 1, n, dtype=torch.int32, device=dev)
        par[off[:-1].long()] = -1
        tok = torch.arange(N, dtype=torch.int32, device=dev) % V
        tau = torch.full((B,), 0.3, device=dev)
        a = asv.verify(x, head, tok, par, off, tau, workspace=ws)
        b = asv.verify(x, head, tok, par, off, tau)
        torch.cuda.synchronize()
        for f in ("row_max", "row_lse", "row_argmax", "accept", "accepted_path", "bonus_token"):
            assert torch.equal(getattr(a, f), getattr(b, f)), f
