"""The entry points of the 8-bit LM head and of the sampling rules on the host: struct layouts, sizes and
refusals, none of which needs a GPU (a call that is refused enqueues nothing; the pointers here are never
read)."""

import ctypes

import pytest

import paper_2609_02897_amd as asv
from paper_2609_02897_amd import _abi, _build
from test_host_checks import _run_host_check

OK, EINVAL, EWORKSPACE = asv.ASV_OK, asv.ASV_EINVAL, asv.ASV_EWORKSPACE
FP8 = _abi.W_FP8
BIG = 1 << 40                      # between the fake arrays, so that none overlap


@pytest.fixture(scope="module")
def lib():
    if not _build.is_built():
        _build.build_library()
    return asv.load()


def _u64(f, *args):
    out = ctypes.c_uint64(0)
    return f(*args, ctypes.byref(out)), out.value


def test_struct_layouts():
    # 4 ints, 3 pointers, an int64
    assert ctypes.sizeof(_abi.AsvLogitsArgs) == 16 + 3 * 8 + 8
    # 5 pointers, an int64, a pointer
    assert ctypes.sizeof(_abi.AsvLogitRules) == 56
    # 4 ints, 2 pointers, 2 int64, 3 pointers, the rules
    assert ctypes.sizeof(_abi.AsvAdjustArgs) == 16 + 2 * 8 + 2 * 8 + 3 * 8 + 56
    # 4 ints, 5 pointers
    assert ctypes.sizeof(_abi.AsvCountsArgs) == 16 + 5 * 8


def test_codes_lie_in_lds_without_conflicts(tmp_path):
    _run_host_check(tmp_path, "q8_swizzle_check")


def test_packed_bytes(lib):
    for V, H in ((1, 64), (256, 128), (257, 192), (151936, 4096), (40003, 2880)):
        rc, n = _u64(lib.asv_fp8_lm_head_bytes, V, H)
        S = -(-V // 256)
        assert rc == OK and n == S * 256 * H + 2 * S * (-(-H // 512) * 4)
    # the codes are addressed with 32 bits
    assert _u64(lib.asv_fp8_lm_head_bytes, 256 * 1023, 1 << 14)[0] == OK
    for V, H in ((0, 64), (-1, 64), (10, 0), (10, 63), (10, 96), (10, (1 << 20) + 64), (256 * 1024, 1 << 14),
                 (1 << 30, 4096)):
        assert _u64(lib.asv_fp8_lm_head_bytes, V, H)[0] == EINVAL, (V, H)
    assert lib.asv_fp8_lm_head_bytes(256, 64, None) == EINVAL


def test_pack_refusals(lib):
    V, H, w, p, sc = 300, 128, BIG, 2 * BIG, 3 * BIG
    n = _u64(lib.asv_fp8_lm_head_bytes, V, H)[1]
    bad = [(None, V, H, p, n), (w, V, H, None, n), (w + 8, V, H, p, n), (w, V, H, p + 8, n),
           (w, V, H, p, n - 1), (w, 0, H, p, n), (w, V, 100, p, n), (w, V, H, w, n),
           (w, V, H, w + 256, n)]
    for a in bad:
        assert lib.asv_quantize_lm_head(*a, None) == EINVAL, a
        assert lib.asv_pack_fp8_lm_head(a[0], sc, *a[1:], None) == EINVAL, a
    assert lib.asv_pack_fp8_lm_head(w, None, V, H, p, n, None) == EINVAL
    assert lib.asv_pack_fp8_lm_head(w, p + 16, V, H, p, n, None) == EINVAL


def test_workspaces_never_fall(lib):
    """A workspace for a larger batch or vocabulary serves a smaller one."""
    H = 64
    for V in (1, 300, 20001, 65537, 140001, 151936):
        last = 0
        for N in (1, 2, 63, 64, 65, 128, 129, 300, 512, 513, 2000):
            rc, n = _u64(lib.asv_verify_ruled_workspace_bytes, 1, N, H, V, FP8)
            assert rc == OK and n >= last, (N, V)
            last = n
            rc, n = _u64(lib.asv_logits_workspace_bytes, N, H, V)
            assert rc == OK and n >= 2 * N * H
    for N in (1, 64, 65, 300):
        for B in (1, N):
            last = 0
            for V in list(range(1, 2000, 37)) + list(range(2000, 300000, 3333)):
                rc, n = _u64(lib.asv_verify_ruled_workspace_bytes, B, N, H, V, FP8)
                assert rc == OK and n >= last, (N, V)
                last = n
    # the bf16 layouts need what asv_verify needs
    for layout in (0, 1):
        assert _u64(lib.asv_verify_ruled_workspace_bytes, 3, 70, 128, 5000, layout) == \
            _u64(lib.asv_workspace_bytes, 3, 70, 128, 5000)
    f = lib.asv_verify_ruled_workspace_bytes
    for a in ((-1, 5, 64, 10, FP8), (1, 0, 64, 10, FP8), (6, 5, 64, 10, FP8), (1, 5, 32, 10, FP8),
              (1, 5, 64, 0, FP8), (1, 5, 64, 10, 3), (1, 5, 64, 10, -1), (1, 5, 1 << 14, 256 * 1024, FP8)):
        assert _u64(f, *a)[0] == EINVAL, a
    assert f(1, 5, 64, 10, FP8, None) == EINVAL
    assert _u64(lib.asv_logits_workspace_bytes, -1, 64, 10)[0] == EINVAL
    assert _u64(lib.asv_logits_workspace_bytes, 5, 65, 10)[0] == EINVAL


def test_logits_refusals(lib):
    def call(ws=4 * BIG, short=0, **kw):
        a = _abi.AsvLogitsArgs()
        a.N, a.H, a.V, a.out_type = 5, 128, 300, _abi.F32
        a.hidden, a.w, a.out, a.out_pitch = BIG, 2 * BIG, 3 * BIG, 300
        for k, v in kw.items():
            setattr(a, k, v)
        need = _u64(lib.asv_logits_workspace_bytes, 5, 128, 300)[1]
        return lib.asv_lm_head_logits(ctypes.byref(a), ws, need - short, None)

    for kw in (dict(N=-1), dict(H=100), dict(V=0), dict(out_type=3), dict(out_type=-1), dict(hidden=None),
               dict(w=None), dict(out=None), dict(out_pitch=299), dict(hidden=BIG + 2),
               dict(w=2 * BIG + 4), dict(out=3 * BIG + 2), dict(out=3 * BIG + 1, out_type=_abi.BF16)):
        assert call(**kw) == EINVAL, kw
    assert lib.asv_lm_head_logits(None, 4 * BIG, 1 << 20, None) == EINVAL
    for kw in (dict(ws=None), dict(ws=4 * BIG + 16), dict(short=1)):
        assert call(**kw) == EWORKSPACE, kw
    assert call(N=0, hidden=None, w=None, out=None) == OK


def _rules(**kw):
    r = _abi.AsvLogitRules()
    for k, v in kw.items():
        setattr(r, k, v)
    return r


BAD_RULES = [dict(counts=BIG + 1), dict(repetition=BIG + 2), dict(presence=BIG + 3), dict(frequency=BIG + 1),
             dict(bias=BIG + 2), dict(allowed=BIG + 1), dict(bias=BIG, bias_pitch=299),
             dict(bias=BIG, bias_pitch=-300)]


def test_verify_refusals(lib):
    def args(**kw):
        a = _abi.AsvVerifyArgs()
        a.B, a.N, a.H, a.V, a.w_lm_layout = 2, 9, 128, 300, FP8
        for i, f in enumerate(("hidden", "w_lm", "draft_tok", "parent", "req_offsets", "tau", "row_max",
                               "row_lse", "row_argmax", "drafted_logit", "accept", "accepted_len",
                               "bonus_token", "accepted_path", "req_status")):
            setattr(a, f, (i + 1) * BIG)
        a.params = asv.make_params()
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    def call(rules=None, ws=90 * BIG, short=0, **kw):
        a = args(**kw)
        need = max(_u64(lib.asv_verify_ruled_workspace_bytes, a.B, a.N, a.H, a.V, a.w_lm_layout)[1], 256)
        return lib.asv_verify_ruled(ctypes.byref(a), rules and ctypes.byref(rules), ws, need - short,
                                    None)

    for kw in (dict(H=100), dict(V=0), dict(w_lm_layout=3), dict(hidden=None), dict(w_lm=None),
               dict(w_lm=2 * BIG + 8), dict(hidden=BIG + 8), dict(row_max=None), dict(req_status=None),
               dict(params=asv.make_params(temperature=0.0)),
               dict(rules=_rules(repetition=BIG), N=65536),
               dict(rules=_rules(repetition=BIG), N=65536, w_lm_layout=1)):
        assert call(**kw) == EINVAL, kw
    for kw in BAD_RULES:
        assert call(rules=_rules(**kw)) == EINVAL, kw
        assert call(rules=_rules(**kw), w_lm_layout=0) == EINVAL, kw
    for kw in (dict(ws=None), dict(ws=90 * BIG + 8), dict(short=1)):
        assert call(**kw) == EWORKSPACE, kw
    assert lib.asv_verify_ruled(None, None, BIG, 1 << 20, None) == EINVAL
    # asv_verify knows no 8-bit weight
    assert lib.asv_verify(ctypes.byref(args()), 90 * BIG, 1 << 30, None) == EINVAL


def test_adjust_refusals(lib):
    def call(rules=None, **kw):
        a = _abi.AsvAdjustArgs()
        a.B, a.N, a.V, a.type = 2, 9, 300, _abi.F32
        a.in_, a.out, a.in_pitch, a.out_pitch = BIG, 2 * BIG, 300, 300
        a.req_offsets, a.parent, a.draft_tok = 3 * BIG, 4 * BIG, 5 * BIG
        for k, v in kw.items():
            setattr(a, k, v)
        if rules:
            a.rules = rules
        return lib.asv_adjust_logits(ctypes.byref(a), None)

    for kw in (dict(B=-1), dict(B=10), dict(B=0), dict(V=0), dict(V=1 << 30), dict(N=1 << 30),
               dict(type=3), dict(in_=None), dict(out=None), dict(in_pitch=299), dict(out_pitch=299),
               dict(in_=BIG + 2), dict(out=2 * BIG + 1), dict(parent=None), dict(draft_tok=None),
               dict(req_offsets=None), dict(req_offsets=None, parent=None, draft_tok=None),
               dict(req_offsets=3 * BIG + 2), dict(parent=4 * BIG + 1), dict(draft_tok=5 * BIG + 2),
               dict(out=BIG, out_pitch=304), dict(out=BIG + 1200), dict(out=BIG - 1200)):
        assert call(**kw) == EINVAL, kw
    for kw in BAD_RULES:
        assert call(rules=_rules(**kw)) == EINVAL, kw
    assert lib.asv_adjust_logits(None, None) == EINVAL
    assert call(B=0, N=0, in_=None, out=None) == OK


def test_counts_refusals(lib):
    def call(**kw):
        a = _abi.AsvCountsArgs()
        a.B, a.T, a.V, a.add = 2, 9, 300, 0
        a.tok, a.tok_offsets, a.counts, a.req_status = BIG, 2 * BIG, 3 * BIG, 4 * BIG
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.asv_token_counts(ctypes.byref(a), None)

    for kw in (dict(B=-1), dict(T=-1), dict(V=0), dict(V=1 << 30), dict(add=2), dict(add=-1), dict(tok=None),
               dict(tok_offsets=None), dict(counts=None), dict(req_status=None),
               dict(counts=3 * BIG + 2), dict(tok=BIG + 1), dict(tok_offsets=2 * BIG + 2),
               dict(prompt_len=5 * BIG + 1), dict(req_status=4 * BIG + 2)):
        assert call(**kw) == EINVAL, kw
    assert lib.asv_token_counts(None, None) == EINVAL
    assert call(B=0, T=0, tok=None, tok_offsets=None, counts=None, req_status=None) == OK


def test_binding_refuses_cpu_tensors_and_other_types():
    torch = pytest.importorskip("torch")
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)             # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)               # noqa: E731
    with pytest.raises(ValueError, match="GPU"):
        asv.quantize_lm_head(bf(300, 64))
    with pytest.raises(ValueError, match="GPU"):
        asv.pack_lm_head_fp8(bf(300, 64).to(torch.float8_e4m3fn), torch.ones((3, 1), dtype=torch.uint8))
    with pytest.raises(ValueError, match="GPU"):
        asv.lm_head_logits(bf(3, 64), asv.PackedLmHead(torch.zeros(8, dtype=torch.uint8), 300, 64, "fp8"))
    with pytest.raises(ValueError, match="GPU"):
        asv.adjust_logits(torch.zeros(3, 300), asv.LogitRules())
    with pytest.raises(ValueError, match="GPU"):
        asv.token_counts(i32(5), i32(2), 300)
    with pytest.raises(TypeError):
        asv.adjust_logits(torch.zeros(3, 300, dtype=torch.float64), asv.LogitRules())
    with pytest.raises(ValueError, match="both or neither"):
        asv.adjust_logits(torch.zeros(3, 300), asv.LogitRules(), parent=i32(3))
    with pytest.raises(ValueError, match="req_offsets"):
        asv.adjust_logits(torch.zeros(3, 300), asv.LogitRules(), parent=i32(3), draft_tok=i32(3))
