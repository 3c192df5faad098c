"""Sampling rules against float64: the history table, the rules on logits in memory, and verification with
rules on either weight."""

import numpy as np
import pytest

import oracle
import rules_oracle as ro
from harness import compare, to_host
from workloads import bf16_weights, build_tree, custom_workload

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


def _t(x, dev):
    import torch
    return torch.from_numpy(np.array(x, order="C")).to(dev)


def _bf16(bits, dev):
    import torch
    return _t(np.asarray(bits, dtype=np.uint16).view(np.int16), dev).view(torch.bfloat16)


# ---------------------------------------------------------------------------- history table

def _table(tok, off, prompt, V):
    out = np.zeros((len(off) - 1, V), dtype=np.int64)
    for b in range(len(off) - 1):
        seen = np.zeros(V, dtype=bool)
        for i, t in enumerate(tok[off[b]:off[b + 1]]):
            if not 0 <= t < V:
                continue
            if prompt is not None and i < prompt[b]:
                seen[t] = True
            else:
                out[b, t] += 1
        out[b] += ro.PROMPT * seen
    return out


@pytest.mark.parametrize("V", [1, 31, 1000, 8192, 8193, 20001])
@pytest.mark.parametrize("lens", [[0], [1], [5, 0, 700], [3000, 1, 64, 65]])
def test_token_counts(asv, dev, V, lens):
    rng = np.random.default_rng([V, len(lens), sum(lens)])
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    tok = (rng.random(off[-1]) ** 4 * V).astype(np.int32)
    prompt = np.array([rng.integers(0, n + 1) for n in lens], dtype=np.int32)
    for p in (prompt, None):
        c, st = asv.token_counts(_t(tok, dev), _t(off, dev), V, None if p is None else _t(p, dev))
        assert np.array_equal(c.cpu().numpy(), _table(tok, off, p, V)) and not st.cpu().numpy().any()
    # more tokens for the same table, twice
    c, _ = asv.token_counts(_t(tok, dev), _t(off, dev), V, _t(prompt, dev))
    for _ in range(2):
        asv.token_counts(_t(tok, dev), _t(off, dev), V, counts=c)
    want = _table(tok, off, prompt, V) + 2 * _table(tok, off, None, V)
    assert np.array_equal(c.cpu().numpy(), want)
    # a prompt added to a table that knows it
    asv.token_counts(_t(tok, dev), _t(off, dev), V, _t(np.array(lens, dtype=np.int32), dev), counts=c)
    known = _table(tok, off, np.array(lens), V) | want
    assert np.array_equal(c.cpu().numpy(), known)


def test_token_counts_of_bad_lists(asv, dev):
    V = 50
    tok = np.array([1, -1, 50, 1, 2**31 - 1, 7, 8], dtype=np.int32)
    c, st = asv.token_counts(_t(tok, dev), _t(np.array([0, 3, 5, 7], np.int32), dev), V)
    assert list(st.cpu()) == [asv.RS_BAD_TOKEN, asv.RS_BAD_TOKEN, 0]
    assert np.array_equal(c.cpu().numpy(), _table(tok, [0, 3, 5, 7], None, V))
    for off in ([0, 8, 3, 5], [-1, 3, 2, 100], [5, 7, 7, 2]):
        c, st = asv.token_counts(_t(tok, dev), _t(np.array(off, np.int32), dev), V)
        for b in range(3):
            bad = off[b] < 0 or off[b + 1] < off[b] or off[b + 1] > 7
            assert bool(st[b].item() & asv.RS_BAD_OFFSETS) == bad
            if bad:
                assert not c[b].any()
    # prompt lengths past the list, and below zero
    c, _ = asv.token_counts(_t(tok[3:4], dev), _t(np.array([0, 1], np.int32), dev), V,
                            _t(np.array([9], np.int32), dev))
    assert c[0, 1].item() == asv.COUNT_PROMPT
    c, _ = asv.token_counts(_t(tok[3:4], dev), _t(np.array([0, 1], np.int32), dev), V,
                            _t(np.array([-9], np.int32), dev))
    assert c[0, 1].item() == 1


# ---------------------------------------------------------------------------- rules in memory

ALL = ("counts", "repetition", "presence", "frequency", "bias", "allowed")


def _rules(rng, B, N, V, names=ALL, shared_bias=False, empty_rows=True):
    counts = np.where(rng.random((B, V)) < 0.1, rng.integers(1, 5, (B, V)), 0)
    counts = counts + ro.PROMPT * (rng.random((B, V)) < 0.1)
    bias = np.where(rng.random((B, V)) < 0.1, 3 * rng.standard_normal((B, V)), 0.0)
    bias = np.where(rng.random((B, V)) < 0.02, -np.inf, bias).astype(np.float32)
    words = -(-V // 32)
    allowed = rng.integers(0, 2**32, (N, words), dtype=np.uint64).astype(np.uint32)
    allowed[rng.random(N) < 0.3] = 0xffffffff
    if empty_rows and N > 3:
        allowed[rng.integers(0, N)] = 0
        allowed[rng.integers(0, N), :] = 1 << 5      # one id of each word
    r = dict(counts=counts.astype(np.int32), repetition=(0.8 + rng.random(B)).astype(np.float32),
             presence=rng.standard_normal(B).astype(np.float32),
             frequency=rng.random(B).astype(np.float32),
             bias=bias[0] if shared_bias else bias, allowed=allowed.view(np.int32))
    return {k: r[k] if k in names else None for k in ALL}


def _dev_rules(asv, r, dev):
    return asv.LogitRules(**{k: None if v is None else _t(v, dev) for k, v in r.items()})


def _trees(rng, sizes, chain=False):
    parent, off = [], [0]
    for n in sizes:
        lo = off[-1]
        for c in range(n):
            parent.append(-1 if c == 0 else lo + (c - 1 if chain else rng.integers(max(0, c - 5), c)))
        off.append(lo + n)
    return np.array(parent, dtype=np.int32), np.array(off, dtype=np.int32)


def _check(got, z, r, dtype, off=None, parent=None, tok=None):
    """A ruled logit is at most five fp32 operations on z: a division or product, a product and two
    additions in the penalty (fused or not), the difference, the bias. Each is off by at most 2^-24 of its
    result, and no intermediate result is larger than M = |z| max(rep, 1 / rep) + |presence| + frequency g +
    |bias|: 5 * 2^-24 M, and half a step of the type."""
    want = ro.ruled(z, r, off, parent, tok)
    hidden = {**r, "allowed": None, "bias": None}
    no = {"frequency": None, "presence": None}
    M = np.abs(z) * 4 + np.abs(ro.ruled(np.abs(z), {**hidden, **no}, off, parent, tok))
    for k in ("presence", "frequency"):
        if r[k] is not None:
            one = {**hidden, **no, "repetition": None, k: -np.abs(r[k])}
            M = M + ro.ruled(0 * z, one, off, parent, tok)
    if r["bias"] is not None:
        M = M + np.abs(ro.ruled(0 * z, {"bias": np.where(np.isfinite(r["bias"]), r["bias"], 0)}, off))
    tol = 5 * 2.0 ** -24 * M
    fin = np.isfinite(want)
    half = {"float32": 0.0, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dtype]
    tol = tol * (1 + half) + half * np.abs(np.where(fin, want, 0)) + (2.0 ** -25 if dtype == "float16" else 0)
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    assert np.array_equal(got[~fin], want[~fin], equal_nan=True)
    bad = np.argwhere(fin & ~(np.abs(got - np.where(fin, want, 0)) <= tol))
    assert len(bad) == 0, (bad[:4], got[tuple(bad[0])], want[tuple(bad[0])])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [1, 7, 32, 1000, 1023, 4100])
@pytest.mark.parametrize("tree", [None, [1], [3, 1, 20, 9], [70]])
def test_adjust(asv, dev, dtype, V, tree):
    import torch
    rng = np.random.default_rng([V, 0 if tree is None else sum(tree)])
    parent, off = _trees(rng, tree) if tree else (None, None)
    N = 11 if tree is None else len(parent)
    B = N if tree is None else len(tree)
    tok = None if tree is None else (rng.random(N) ** 3 * V).astype(np.int32)
    x = _t((4 * rng.standard_normal((N, V))).astype(np.float32), dev).to(getattr(torch, dtype))
    z = x.double().cpu().numpy()
    tree_d = [None if a is None else _t(a, dev) for a in (off, parent, tok)]
    sets = [ALL, (), ("allowed",), ("bias",), ("repetition",), ("counts", "frequency"), ALL]
    for k, names in enumerate(sets):
        r = _rules(rng, B, N, V, names, shared_bias=k == 3)
        got = asv.adjust_logits(x, _dev_rules(asv, r, dev), *tree_d)
        _check(got.double().cpu().numpy(), z, r, dtype, off, parent, tok)
    # in place; and no tree's tokens where only the offsets are given
    same = asv.adjust_logits(x.clone(), _dev_rules(asv, r, dev), *tree_d)
    y = x.clone()
    assert asv.adjust_logits(y, _dev_rules(asv, r, dev), *tree_d, out=y) is y
    assert torch.equal(y, same)
    if tree:
        got = asv.adjust_logits(x, _dev_rules(asv, r, dev), tree_d[0])
        _check(got.double().cpu().numpy(), z, r, dtype, off)


@pytest.mark.parametrize("pitch", [301, 304, 320])
def test_adjust_rows_apart(asv, dev, pitch):
    """Rows apart from each other, at odd addresses; what lies between them stays."""
    import torch
    N, V = 21, 300
    rng = np.random.default_rng(pitch)
    r = _rules(rng, N, N, V)
    d = _dev_rules(asv, r, dev)
    x = torch.randn((N, V), device=dev)
    bias = torch.full((N, V + 5), 9.0, device=dev)[:, :V]
    bias.copy_(d.bias)
    for dtype in (torch.float32, torch.bfloat16):
        want = asv.adjust_logits(x.to(dtype), d)
        for first in (0, 1):
            buf = torch.full((3, N * pitch + 2), 7.0, dtype=dtype, device=dev)
            at = [b[first:first + N * pitch].view(N, pitch)[:, :V] for b in buf]
            at[0].copy_(x)
            assert torch.equal(asv.adjust_logits(at[0], d._replace(bias=bias), out=at[1]), want)
            asv.adjust_logits(at[0], d, out=at[0])
            assert torch.equal(at[0], want)
            at[0].fill_(7.0)
            at[1].fill_(7.0)
            assert bool((buf == 7.0).all())


def test_adjust_masked_specials(asv, dev):
    """NaN and infinities where the mask forbids give -inf, and pass through where it allows; bits
    past V mean nothing."""
    import torch
    V = 37
    x = torch.tensor([[float("nan"), float("inf"), -float("inf"), 1.0] + [0.0] * (V - 4)] * 3,
                     device=dev)
    allowed = torch.tensor([[0, 0], [-1, -1], [0b0100, -32]], dtype=torch.int32, device=dev)
    got = asv.adjust_logits(x, asv.LogitRules(allowed=allowed)).cpu()
    assert bool((got[0] == -float("inf")).all())
    assert torch.equal(got[1].nan_to_num(nan=5.0), x[1].cpu().nan_to_num(nan=5.0))
    assert got[2, 2] == -float("inf") and bool((got[2, :32] == -float("inf")).all())
    assert bool((got[2, 32:] == -float("inf")).all())     # -32: bits 0 .. 4 of the second word are clear


def test_adjust_long_paths(asv, dev):
    """A chain longer than what is staged, with one token many times over, and a row group that starts inside
    a request."""
    import torch
    n, V = 700, 600
    parent, off = _trees(None, [n], chain=True)
    rng = np.random.default_rng(2)
    tok = np.where(rng.random(n) < 0.6, 17, rng.integers(0, V, n)).astype(np.int32)
    r = dict.fromkeys(ALL)
    r.update(frequency=np.array([0.25], np.float32), presence=np.array([1.0], np.float32),
             repetition=np.array([1.5], np.float32))
    z = rng.standard_normal((n, V)).astype(np.float32)
    got = asv.adjust_logits(_t(z, dev), _dev_rules(asv, r, dev), _t(off, dev), _t(parent, dev), _t(tok, dev))
    _check(got.double().cpu().numpy(), z.astype(np.float64), r, "float32", off, parent, tok)


def test_adjust_malformed_trees_stay_in_bounds(asv, dev):
    """Offsets and links that no tree has: the call returns, rows of no request are copied."""
    import torch
    N, V = 30, 90
    x = torch.randn((N, V), device=dev)
    rng = np.random.default_rng(1)
    r = _rules(rng, 2, N, V, empty_rows=False)
    d = _dev_rules(asv, r, dev)
    tok = _t(rng.integers(-5, V + 5, N).astype(np.int32), dev)
    for off in ([0, 12, 40], [5, 12, 30], [0, 25, 9], [-7, 10, 30], [30, 30, 30]):
        for parent in (np.full(N, 2**31 - 1), np.arange(N), np.full(N, -2**31), np.arange(N) + 1):
            got = asv.adjust_logits(x, d, _t(np.array(off, np.int32), dev), _t(parent.astype(np.int32), dev),
                                    tok)
            torch.cuda.synchronize()
            inside = np.zeros(N, dtype=bool)
            for lo, hi in zip(off, off[1:]):
                if lo >= 0:
                    inside[lo:max(lo, min(hi, N))] = True
            keep = torch.from_numpy(~inside).to(dev)
            assert torch.equal(got[keep], x[keep])


# ---------------------------------------------------------------------------- verification

def _workload(kind, n_req, H, V, seed):
    rng = np.random.default_rng([seed, 7])
    trees = [build_tree(kind, rng, b) for b in range(n_req)]
    return custom_workload("ruled", H, V, trees, 0.2, seed=seed, w_std=0.09)


def _draft_under_rules(w, z, r, rng):
    """Drafted tokens, parents before children: the parent's ruled top, one of its best, an ancestor's token, a
    banned one or any."""
    V = z.shape[1]
    w.draft_tok = np.zeros(w.N, dtype=np.int32)
    off = np.asarray(w.req_offsets)
    for c in range(w.N):
        p = int(w.parent[c])
        if p < 0:
            continue
        b = int(np.searchsorted(off, c, side="right") - 1)
        # the parent's row alone, under the rules
        sub = {k: (v if v is None or k != "allowed" else v[[p]]) for k, v in r.items()}
        for k in ("counts", "repetition", "presence", "frequency"):
            sub[k] = None if r[k] is None else r[k][[b]]
        if r["bias"] is not None and r["bias"].ndim == 2:
            sub["bias"] = r["bias"][[b]]
        path = ro.path_tokens(p, w.parent, w.draft_tok)
        par = np.array([-1] + list(range(len(path))), dtype=np.int64)
        zz = np.vstack([z[[p]]] * len(par))
        if sub["allowed"] is not None:
            sub["allowed"] = np.vstack([sub["allowed"]] * len(par))
        row = ro.ruled(zz, sub, np.array([0, len(par)]), par, np.array([0] + path[::-1]))[-1]
        u = rng.random()
        best = np.argsort(-row, kind="stable")
        if u < 0.5:
            t = best[0]
        elif u < 0.7:
            t = best[min(rng.integers(0, 6), V - 1)]
        elif u < 0.85 and path:
            t = path[rng.integers(0, len(path))]
        else:
            t = rng.integers(0, V)
        w.draft_tok[c] = t


def _run(asv, dev, w, W, r, tau, head, **kw):
    import torch
    hidden, wt = _bf16(w.hidden, dev), _bf16(W, dev)
    head = {"row": lambda: wt, "packed": lambda: asv.pack_lm_head(wt),
            "fp8": lambda: asv.quantize_lm_head(wt)}[head]()
    out = asv.verify(hidden, head, _t(w.draft_tok.astype(np.int32), dev),
                     _t(w.parent.astype(np.int32), dev), _t(w.req_offsets.astype(np.int32), dev),
                     _t(tau, dev), rules=None if r is None else _dev_rules(asv, r, dev), **kw)
    torch.cuda.synchronize()
    return to_host(out)


def _values(w, W, head):
    x, v = oracle.widen_bf16(w.hidden), oracle.widen_bf16(W)
    if head == "fp8":
        x, v = ro.quantise(x, 1)[2], ro.quantise(v, 128)[2]
    return x @ v.T


def _compare(w, ref, got):
    """harness.compare on the finite values; rows and tokens that the rules leave nothing exactly."""
    empty = np.isneginf(ref["row_max"])
    nonroot = np.asarray(w.parent) >= 0
    assert np.array_equal(np.isneginf(got["row_max"]), empty)
    assert np.array_equal(np.isneginf(got["row_lse"]), empty)
    assert np.all(got["row_argmax"][empty] == -1)
    ban = np.isneginf(ref["drafted_logit"]) & nonroot
    assert np.array_equal(np.isneginf(got["drafted_logit"][nonroot]), ban[nonroot])
    assert not got["accept"][ban].any()
    fix = lambda a, m: np.where(m, 0.0, a)      # noqa: E731
    ref2, got2 = dict(ref), dict(got)
    for d in (ref2, got2):
        d["row_max"], d["row_lse"] = fix(d["row_max"], empty), fix(d["row_lse"], empty)
        d["drafted_logit"] = fix(d["drafted_logit"], ban | ~nonroot)
    compare_w = type("W", (), dict(N=w.N, B=w.B, parent=np.asarray(w.parent), draft_tok=w.draft_tok,
                                   req_offsets=w.req_offsets))
    # margins of banned tokens and empty rows are no near-ties
    ref2["row_max"] = ref2["row_max"] + fix(0.0 * ref["tau_node"], False)
    rep = compare(compare_w, ref2, got2)
    return rep


CASES = [("tiny", 1, 64, 300, "packed"), ("eagle60", 1, 128, 2001, "packed"),
         ("eagle60", 2, 128, 2000, "row"), ("adaptive", 4, 192, 1300, "packed"),
         ("level8x8", 7, 64, 1030, "row"), ("tiny", 3, 64, 2600, "fp8"), ("eagle60", 1, 192, 3000, "fp8"),
         ("level8x8", 2, 128, 1025, "fp8"), ("adaptive", 6, 320, 900, "fp8")]


@pytest.mark.parametrize("kind,n_req,H,V,head", CASES)
def test_verify_with_rules(asv, dev, kind, n_req, H, V, head):
    w = _workload(kind, n_req, H, V, 11)
    W = bf16_weights(V, H, 0.09, 31)
    z = _values(w, W, head)
    rng = np.random.default_rng([n_req, V])
    for names in (ALL, ("allowed",), ("counts", "repetition", "presence", "frequency")):
        r = _rules(rng, w.B, w.N, V, names, shared_bias=n_req % 2 == 0)
        _draft_under_rules(w, z, r, rng)
        tau = rng.choice([0.0, 0.05, 0.3, 1.0], w.B).astype(np.float32)
        zr = ro.ruled(z, r, w.req_offsets, w.parent, w.draft_tok)
        ref = ro.verify(zr, w, tau)
        got = _run(asv, dev, w, W, r, tau, head)
        _compare(w, ref, got)


@pytest.mark.parametrize("head", ["row", "packed"])
def test_no_rules_is_verify(asv, dev, head):
    """LogitRules without a rule, and rules that change nothing, give verify's results."""
    w = _workload("adaptive", 5, 128, 1500, 3)
    W = bf16_weights(w.V, w.H, 0.09, 12)
    w.with_drafts(oracle.row_top8(_values(w, W, head)))
    nonroot = w.parent >= 0
    base = _run(asv, dev, w, W, None, w.tau, head)
    one = dict.fromkeys(ALL)
    words = -(-w.V // 32)
    neutral = dict(counts=np.ones((w.B, w.V), np.int32), repetition=np.ones(w.B, np.float32),
                   presence=np.zeros(w.B, np.float32), frequency=np.zeros(w.B, np.float32),
                   bias=np.zeros(w.V, np.float32), allowed=np.full((w.N, words), -1, np.int32))
    for r in (one, neutral):
        got = _run(asv, dev, w, W, r, w.tau, head)
        for k, v in base.items():
            if v is None:
                continue
            sel = nonroot if k == "drafted_logit" else slice(None)
            if k == "row_lse":          # the ids of a record may be cut elsewhere: sums in another order
                assert np.allclose(got[k], v, rtol=0, atol=2.0 ** -24 * (w.V + 2) * np.abs(v).max())
            else:
                assert np.array_equal(got[k][sel], v[sel]), k


def test_dead_ends(asv, dev):
    """A grammar that leaves a row nothing ends the walk there with the bonus -1; a banned token is not
    accepted at tau = 0; one allowed id is the bonus whatever its logit."""
    H, V, n = 64, 700, 4
    w = custom_workload("dead", H, V, [np.array([-1, 0, 1, 2])] * 3, 0.0, seed=2, w_std=0.09)
    W = bf16_weights(V, H, 0.09, 5)
    z = _values(w, W, "packed")
    w.draft_tok = np.arange(w.N).astype(np.int32) * 7 % V
    allowed = np.full((w.N, -(-V // 32)), -1, dtype=np.int32)
    allowed[1] = 0                                        # request 0 dies below its first node
    allowed[n] = 0                                        # request 1: only id 321 at the root
    allowed[n, 321 // 32] = 1 << (321 % 32)
    tau = np.zeros(3, np.float32)
    for head in ("packed", "fp8"):
        got = _run(asv, dev, w, W, {**dict.fromkeys(ALL), "allowed": allowed}, tau, head)
        assert list(got["accepted_len"]) == [1, 0, 3]
        assert got["bonus_token"][0] == -1 and got["bonus_token"][1] == 321
        assert list(got["accept"][:n]) == [1, 1, 0, 1] and got["accept"][n + 1] == 0
        assert not got["req_status"].any()


def test_malformed_requests_report_as_in_verify(asv, dev):
    w = _workload("tiny", 3, 64, 300, 4)
    W = bf16_weights(w.V, w.H, 0.09, 5)
    rng = np.random.default_rng(3)
    w.draft_tok = rng.integers(0, w.V, w.N).astype(np.int32)
    r = _rules(rng, w.B, w.N, w.V)
    base = w.parent.copy()
    lo = int(w.req_offsets[1])
    for at, value, bit in ((lo, 3, asv.RS_BAD_ROOT), (lo + 1, lo + 5, asv.RS_BAD_PARENT),
                           (lo + 1, -1, asv.RS_BAD_PARENT)):
        w.parent = base.copy()
        w.parent[at] = value
        for head in ("packed", "fp8"):
            got = _run(asv, dev, w, W, r, w.tau, head)
            assert list(got["req_status"]) == [0, bit, 0]
    w.parent = base
    w.draft_tok[lo + 1] = w.V
    got = _run(asv, dev, w, W, r, w.tau, "fp8")
    assert list(got["req_status"]) == [0, asv.RS_BAD_TOKEN, 0] and got["bonus_token"][1] == -1


def test_long_chain_in_tiles(asv, dev):
    """A path over several row tiles, longer than what is staged, with a token many times on it."""
    n, H, V = 600, 64, 500
    w = custom_workload("chain", H, V, [np.arange(-1, n - 1)], 0.2, seed=9, w_std=0.09)
    W = bf16_weights(V, H, 0.09, 6)
    rng = np.random.default_rng(4)
    w.draft_tok = np.where(rng.random(n) < 0.6, 300, rng.integers(0, V, n)).astype(np.int32)
    r = dict.fromkeys(ALL)
    r.update(frequency=np.array([0.01], np.float32), repetition=np.array([1.2], np.float32))
    for head in ("packed", "fp8"):
        z = ro.ruled(_values(w, W, head), r, w.req_offsets, w.parent, w.draft_tok)
        _compare(w, ro.verify(z, w, w.tau), _run(asv, dev, w, W, r, w.tau, head))


def test_more_requests_than_a_workgroup_has_threads(asv, dev):
    """1100 requests of one and two nodes (the unfused finishing step)."""
    sizes = [np.array([-1] + [0] * (b % 2)) for b in range(1100)]
    H, V = 64, 260
    w = custom_workload("many", H, V, sizes, 0.1, seed=6, w_std=0.09)
    W = bf16_weights(V, H, 0.09, 6)
    rng = np.random.default_rng(8)
    r = _rules(rng, w.B, w.N, V)
    for head in ("packed", "fp8"):
        z = _values(w, W, head)
        _draft_under_rules(w, z, r, rng)
        ref = ro.verify(ro.ruled(z, r, w.req_offsets, w.parent, w.draft_tok), w, w.tau)
        _compare(w, ref, _run(asv, dev, w, W, r, w.tau, head))
