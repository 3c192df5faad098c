"""The 8-bit LM head, the sampling rules and the history table as a server runs them: one decoding step
after the other through all of them, captured into graphs that share a workspace, on other streams, from
two threads, and with arrays of more than 2^31 elements."""

import threading

import numpy as np
import pytest

import oracle
import rules_oracle as ro
from test_fp8_head_gpu import _check_logits
from test_rules_gpu import ALL, _bf16, _check, _dev_rules, _rules, _t, _table, _trees
from workloads import bf16_normal, bf16_weights

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


def _same(a, b):
    import torch
    a, b = a.contiguous(), b.contiguous()
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


class Batch:
    """Ragged trees of B requests on a V-id vocabulary, with histories and rules."""

    def __init__(self, asv, dev, sizes, V, H, seed):
        self.rng = np.random.default_rng([seed, V, H])
        self.parent, self.off = _trees(self.rng, sizes)
        self.B, self.N, self.V, self.H = len(sizes), int(self.off[-1]), V, H
        lens = self.rng.integers(0, 200, self.B)
        self.h_off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.hist = (self.rng.random(self.h_off[-1]) ** 3 * V).astype(np.int32)
        self.prompt = (lens // 2).astype(np.int32)
        self.W = bf16_weights(V, H, 0.3, seed)
        self.dev = dev
        self.d_parent, self.d_off = _t(self.parent, dev), _t(self.off, dev)
        self.tau = _t(np.linspace(0.0, 1.0, self.B).astype(np.float32), dev)
        self.head = asv.quantize_lm_head(_bf16(self.W, dev))

    def step(self):
        """Hidden states, drafted tokens and the rules of one step (numpy; without the counts)."""
        r = _rules(self.rng, self.B, self.N, self.V, ALL[1:])
        return bf16_normal(self.rng, (self.N, self.H), 1.0), \
            self.rng.integers(0, self.V, self.N).astype(np.int32), r


SIZES = [[9, 1, 24], [70, 3, 60, 33]]      # one 64-row tile; several row tiles


@pytest.mark.parametrize("sizes", SIZES)
def test_decoding_steps(asv, dev, sizes):
    """Three steps: the table, verification with rules on the 8-bit head, commit, the committed tokens into
    the table; beside them the logits of the same head under the same rules, which the records agree
    with bit for bit."""
    import torch
    b = Batch(asv, dev, sizes, 3001, 192, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                    # not the default stream
        counts, st = asv.token_counts(_t(b.hist, dev), _t(b.h_off, dev), b.V, _t(b.prompt, dev))
        assert not st.cpu().numpy().any()
        table = _table(b.hist, b.h_off, b.prompt, b.V)
        wq = ro.quantise(oracle.widen_bf16(b.W), 128)[2]
        for step in range(3):
            x, tok, r = b.step()
            d_x, d_tok = _bf16(x, dev), _t(tok, dev)
            rules = _dev_rules(asv, r, dev)._replace(counts=counts)
            # bit for bit: the same sums, the same roundings
            z = asv.lm_head_logits(d_x, b.head)
            out = asv.verify(d_x, b.head, d_tok, b.d_parent, b.d_off, b.tau, rules=rules)
            zr = asv.adjust_logits(z, rules, b.d_off, b.d_parent, d_tok)
            assert torch.equal(out.row_max, zr.max(1).values)
            some = out.row_max > -float("inf")
            first = (zr == out.row_max[:, None]).int().argmax(1)
            assert torch.equal(out.row_argmax.long(), torch.where(some, first, -1))
            up = b.d_parent.long().clamp(min=0)
            kid = b.d_parent >= 0
            assert torch.equal(out.drafted_logit[kid], zr[up, d_tok.long()][kid])
            # against the definitions
            xq = ro.quantise(oracle.widen_bf16(x), 1)[2]
            _check_logits(z.double().cpu().numpy(), xq, wq, "float32")
            _check(zr.double().cpu().numpy(), z.double().cpu().numpy(), {**r, "counts": table}, "float32",
                   b.off, b.parent, tok)
            # what was accepted enters the history; an empty row's bonus (-1) does not
            assert not out.req_status.cpu().numpy().any()
            c_off, c_tok, _, _, c_st = asv.commit(b.d_off, d_tok, out.accepted_len, out.accepted_path,
                                                  out.bonus_token)
            _, st = asv.token_counts(c_tok, c_off, b.V, counts=counts)
            new = _table(c_tok.cpu().numpy(), c_off.cpu().numpy(), None, b.V)
            assert new.sum() == int(((c_tok >= 0)[:int(c_off[-1])]).sum())
            table = table + new
            assert np.array_equal(counts.cpu().numpy(), table)
    torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("sizes", SIZES)
def test_two_graphs_that_share_a_workspace(asv, dev, sizes):
    """One graph counts, verifies and counts again, the other writes the logits and adjusts them in place;
    replayed in turn on one workspace with eager work between, they give the eager calls' bits."""
    import torch
    b = Batch(asv, dev, sizes, 2500, 128, 7)
    ws = asv.alloc_workspace(b.B, b.N, b.H, b.V, dev, b.head)
    assert ws.numel() >= asv.logits_workspace_bytes(b.N, b.H, b.V)
    x, tok, r = b.step()
    d_x, d_tok = _bf16(x, dev), _t(tok, dev)
    hist, h_off, prompt = _t(b.hist, dev), _t(b.h_off, dev), _t(b.prompt, dev)
    rules = _dev_rules(asv, r, dev)
    out = asv.alloc_outputs(b.B, b.N, dev, False)
    z = torch.empty((b.N, b.V), dtype=torch.bfloat16, device=dev)
    table = torch.zeros((b.B, b.V), dtype=torch.int32, device=dev)

    def verify(counts, o, w, state):
        asv.token_counts(hist, h_off, b.V, prompt, counts=counts)
        asv.verify(d_x, b.head, d_tok, b.d_parent, b.d_off, b.tau, state=state, out=o, workspace=w,
                   rules=rules._replace(counts=counts))

    def logits(counts, o, w):
        asv.lm_head_logits(d_x, b.head, out=o, workspace=w)
        asv.adjust_logits(o, rules._replace(counts=counts), b.d_off, b.d_parent, d_tok, out=o)

    state = asv.state_init(b.B, device=dev)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        verify(table, out, ws, state)
        logits(table, z, ws)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        verify(table, out, ws, state)
    with torch.cuda.graph(graphs[1]):
        logits(table, z, ws)
    table.zero_()
    state.copy_(asv.state_init(b.B, device=dev))
    want_table, want_state = torch.zeros_like(table), state.clone()
    for _ in range(4):
        x, tok, r = b.step()
        d_x.copy_(_bf16(x, dev))
        d_tok.copy_(_t(tok, dev))
        for dst, src in zip(rules[1:], _dev_rules(asv, r, dev)[1:]):
            dst.copy_(src)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        ref, zz = asv.alloc_outputs(b.B, b.N, dev, False), torch.empty_like(z)
        other = asv.alloc_workspace(b.B, b.N, b.H, b.V, dev, b.head)
        verify(want_table, ref, other, want_state)
        logits(want_table, zz, other)
        torch.cuda.synchronize()
        kid = b.d_parent >= 0
        for f in ref._fields:
            p, q = getattr(ref, f), getattr(out, f)
            if p is None:
                continue
            if f == "drafted_logit":                  # unspecified at roots
                p, q = p[kid], q[kid]
            assert _same(p, q), f
        assert torch.equal(table, want_table) and _same(state, want_state) and _same(z, zz)


def test_two_threads_on_two_streams(asv, dev):
    """Each with its own batch, outputs and workspace."""
    import torch
    work = [Batch(asv, dev, sizes, V, 128, 3) for sizes, V in (([60], 2000), ([40, 50, 60], 1500))]
    args = []
    for b in work:
        x, tok, r = b.step()
        args.append((_bf16(x, dev), _t(tok, dev), _dev_rules(asv, r, dev)))

    def go(k):
        b, (x, tok, rules) = work[k], args[k]
        out = asv.verify(x, b.head, tok, b.d_parent, b.d_off, b.tau, rules=rules)
        z = asv.lm_head_logits(x, b.head)
        return [out.row_max, out.row_lse, out.bonus_token, asv.adjust_logits(z, rules, b.d_off), z]

    want = [go(0), go(1)]
    torch.cuda.synchronize()
    bad = []

    def run(k):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got = go(k)
                s.synchronize()
                if not all(_same(p, q) for p, q in zip(got, want[k])):
                    bad.append(k)

    threads = [threading.Thread(target=run, args=(k,)) for k in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not bad


def test_more_than_2_31_elements(asv, dev):
    """Logits, tables and masks whose last rows lie past 2^31 elements: the last rows are those of a call
    on these rows alone."""
    import torch
    N, V, H, n = 17000, 128256, 64, 40
    g = torch.Generator(device=dev).manual_seed(1)
    w = torch.randn(V, H, device=dev, generator=g).bfloat16()
    x = torch.randn(N, H, device=dev, generator=g).bfloat16()
    head = asv.quantize_lm_head(w)
    z = asv.lm_head_logits(x, head, dtype=torch.bfloat16)
    assert z.numel() > 2 ** 31
    assert torch.equal(z[-n:], asv.lm_head_logits(x[-n:].contiguous(), head, dtype=torch.bfloat16))
    # one token of request b is b, two are 7
    tok = torch.full((3 * N,), 7, dtype=torch.int32, device=dev)
    tok[::3] = torch.arange(N, dtype=torch.int32, device=dev)
    off = 3 * torch.arange(N + 1, dtype=torch.int32, device=dev)
    counts, st = asv.token_counts(tok, off, V)
    assert not st.any() and counts[-1].sum() == 3 and counts[-1, 7] == 2 and counts[-1, N - 1] == 1
    few, _ = asv.token_counts(tok[-3 * n:].contiguous(), off[:n + 1].contiguous(), V)
    assert torch.equal(counts[-n:], few)
    rep = 1.0 + torch.rand(N, device=dev, generator=g)
    allowed = torch.randint(-2 ** 31, 2 ** 31, (N, -(-V // 32)), device=dev, generator=g,
                            dtype=torch.int64).int()
    part = asv.adjust_logits(z[-n:], asv.LogitRules(counts=few, repetition=rep[-n:].contiguous(),
                                                    allowed=allowed[-n:].contiguous()))
    asv.adjust_logits(z, asv.LogitRules(counts=counts, repetition=rep, allowed=allowed), out=z)
    assert torch.equal(z[-n:], part)
    torch.cuda.synchronize()


@pytest.mark.parametrize("N", [5, 70, 300])
def test_codes_past_2_gib(asv, dev, N):
    """The last ids of a head of 2.3 GB of codes: as in a head of these ids alone."""
    import torch
    V, H, first = 140001, 16384, 128 * 1080
    w = torch.randn(V, H, dtype=torch.bfloat16, device=dev)
    x = torch.randn(N, H, dtype=torch.bfloat16, device=dev)
    head = asv.quantize_lm_head(w)
    assert head.data.numel() > 2 ** 31
    z = asv.lm_head_logits(x, head)
    tail = asv.lm_head_logits(x, asv.quantize_lm_head(w[first:]))
    assert torch.equal(z[:, first:], tail)
    start = asv.lm_head_logits(x, asv.quantize_lm_head(w[:1024]))
    assert torch.equal(z[:, :1024], start)


def test_scales_of_a_checkpoint(asv, dev):
    """Every scale byte, on finite codes: q 2^(s - 127); 255 is no number. Where the product of code and
    scale falls below 2^-126 it may be taken as zero."""
    import torch
    H, V = 128, 128 * 256
    rng = np.random.default_rng(2)
    codes = rng.integers(0, 256, (V, H)).astype(np.uint8)
    codes[(codes & 127) == 127] = 1                         # no NaN
    value = ro.E4M3[codes]
    step = 2.0 ** (np.arange(256.0) - 127)
    # past fp32's largest a value is infinite: leave the codes of those blocks below 2
    big = np.arange(V)[:, None] // 128 >= 246
    codes = np.where(big & (np.abs(value) >= 2), 0x38, codes).astype(np.uint8)
    value = ro.E4M3[codes]
    scale = np.arange(256, dtype=np.uint8)[:, None]
    head = asv.pack_lm_head_fp8(_t(codes, dev).view(torch.float8_e4m3fn), _t(scale, dev))
    col = int(rng.integers(0, H))
    w = value[:, col] * np.repeat(step, 128)
    for e in (-60, 0, 100):                                 # one column at a time: every product is exact
        x = np.zeros((1, H))
        x[0, col] = 2.0 ** e
        got = asv.lm_head_logits(_bf16((x.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16), dev),
                                 head)[0].double().cpu().numpy()
        want = w * 2.0 ** e
        nan = np.arange(V) // 128 == 255
        assert np.all(np.isnan(got[nan]))
        inf = ~nan & (np.abs(want) >= 2.0 ** 128)
        assert np.all(np.isinf(got[inf]) | np.isnan(got[inf]))
        tiny = (np.abs(w) < 2.0 ** -126) | (np.abs(want) < 2.0 ** -126)
        ok = ~nan & ~inf
        assert np.array_equal(got[ok & ~tiny], want[ok & ~tiny])
        assert np.all((got[ok & tiny] == want[ok & tiny]) | (got[ok & tiny] == 0) |
                      (np.abs(got[ok & tiny] - want[ok & tiny]) <= 2.0 ** -126 * max(1.0, 2.0 ** e)))


def test_tables_of_many_requests(asv, dev):
    """As many ids a workgroup as its LDS holds, in an odd vocabulary and in one of whole vectors."""
    rng = np.random.default_rng(12)
    lens = rng.integers(0, 60, 700)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    for V in (50001, 40960):
        tok = rng.integers(0, V, off[-1]).astype(np.int32)
        prompt = rng.integers(0, 60, 700).astype(np.int32)
        c, st = asv.token_counts(_t(tok, dev), _t(off, dev), V, _t(prompt, dev))
        assert np.array_equal(c.cpu().numpy(), _table(tok, off, np.minimum(prompt, lens), V))
        assert not st.cpu().numpy().any()


@pytest.mark.parametrize("offsets", [[0, 9, 5, 20], [0, -3, 9, 20], [0, 7, 25, 20], [1, 7, 9, 20], [0, 7, 9, 19],
                                     [0, 0, 9, 20]])
def test_malformed_offsets_on_the_8_bit_head(asv, dev, offsets):
    """The requests report, and the rows give, what they do on the bf16 weight."""
    import torch
    N, B, V, H = 20, 3, 700, 64
    # a power of two an entry, so that the 8-bit head holds the bf16 values
    rng = np.random.default_rng(3)
    pick = lambda *s: ((rng.integers(0, 4, s) + 126 << 7) | (rng.integers(0, 2, s) << 15)).astype(   # noqa: E731
        np.uint16)
    x, w = _bf16(pick(N, H), dev), _bf16(pick(V, H), dev)
    parent = np.array([max(c - 1, -1) if c not in (7, 9) else -1 for c in range(N)], dtype=np.int32)
    args = (_t(rng.integers(0, V, N).astype(np.int32), dev), _t(parent, dev),
            _t(np.array(offsets, np.int32), dev), torch.full((B,), 0.3, device=dev))
    a = asv.verify(x, w, *args)
    for rules in (None, asv.LogitRules(repetition=torch.ones(B, device=dev))):
        b = asv.verify(x, asv.quantize_lm_head(w), *args, rules=rules)
        torch.cuda.synchronize()
        assert a.req_status.any() and torch.equal(a.req_status, b.req_status)
        assert torch.equal(a.accepted_len, b.accepted_len) and torch.equal(a.bonus_token, b.bonus_token)


CUTS = [([60], 20000), ([60], 40003), ([5, 44], 70001), ([64], 100001), ([33], 128256), ([60], 152001),
        ([7, 50], 168003), ([61], 181003), ([20], 200001), ([30, 40, 30], 20000), ([100], 32000),
        ([70, 58], 75003), ([190], 16003), ([90, 100], 67003), ([100, 101, 55], 14001), ([256], 70003),
        ([80, 70, 90, 93], 40003), ([150, 150], 36003), ([500], 18000), ([378], 151936), ([300, 301], 70003)]


@pytest.mark.parametrize("sizes,V", CUTS)
def test_rules_over_every_cut(asv, dev, sizes, V):
    """Weights and hidden states whose products and sums fp32 and both heads hold exactly: verification with
    rules on the bf16 and on the 8-bit head gives the ruled logits' own maxima, argmaxes and drafted logits,
    bit for bit, over every tile family and cut of the ids."""
    import torch
    H, B = 64, len(sizes)
    rng = np.random.default_rng([V, B])
    g = torch.Generator(device=dev).manual_seed(V)
    def exact(*s):                                        # +-1/2, 1, 2 or 4
        return ((2.0 ** torch.randint(-1, 3, s, device=dev, generator=g)) *
                (2 * torch.randint(0, 2, s, device=dev, generator=g) - 1)).bfloat16()
    parent, off = _trees(rng, sizes)
    N = int(off[-1])
    x, w = exact(N, H), exact(V, H)
    parent, off = _t(parent, dev), _t(off, dev)
    tok = torch.randint(0, V, (N,), device=dev, generator=g, dtype=torch.int32)
    tok[N // 3::4] = tok[0]                               # ids that many paths share
    ids = torch.randint(0, V, (B, 500), device=dev, generator=g, dtype=torch.int32)
    counts, _ = asv.token_counts(ids.view(-1), 500 * torch.arange(B + 1, dtype=torch.int32, device=dev), V)
    rules = asv.LogitRules(counts, 1.0 + torch.rand(B, device=dev, generator=g),
                           torch.rand(B, device=dev, generator=g), torch.rand(B, device=dev, generator=g),
                           torch.randn((B, V), device=dev, generator=g),
                           torch.randint(-2 ** 31, 2 ** 31, (N, -(-V // 32)), device=dev, generator=g,
                                         dtype=torch.int64).int())
    head = asv.quantize_lm_head(w)
    zr = asv.adjust_logits(asv.lm_head_logits(x, head), rules, off, parent, tok)
    top = zr.max(1).values
    arg = (zr == top[:, None]).int().argmax(1).int()
    kid = parent >= 0
    drafted = zr[parent.long().clamp(min=0), tok.long()][kid]
    lse = torch.logsumexp(zr.double(), 1)
    tau = torch.full((B,), 0.3, device=dev)
    for weight in (head, w, asv.pack_lm_head(w)):
        out = asv.verify(x, weight, tok, parent, off, tau, rules=rules)
        torch.cuda.synchronize()
        assert not out.req_status.any()
        assert torch.equal(out.row_max, top) and torch.equal(out.row_argmax, arg)
        assert torch.equal(out.drafted_logit[kid], drafted)
        assert bool(((out.row_lse.double() - lse).abs() < 1e-4).all())


def test_refusals_of_the_binding(asv, dev):
    import torch
    V, H, N = 300, 64, 4
    w = torch.zeros((V, H), dtype=torch.bfloat16, device=dev)
    x = torch.zeros((N, H), dtype=torch.bfloat16, device=dev)
    head, i = asv.quantize_lm_head(w), lambda *a: torch.tensor(a, dtype=torch.int32, device=dev)
    z = torch.zeros((N, V), device=dev)
    one = torch.ones(N, device=dev)
    with pytest.raises(TypeError):
        asv.lm_head_logits(x, w)                                        # a bf16 weight
    with pytest.raises(TypeError):
        asv.lm_head_logits(x, asv.pack_lm_head(w))
    with pytest.raises(ValueError):
        asv.lm_head_logits(torch.zeros((N, 128), dtype=torch.bfloat16, device=dev), head)
    with pytest.raises(TypeError):
        asv.lm_head_logits(x, head, dtype=torch.float64)
    with pytest.raises(TypeError):
        asv.lm_head_logits(x, head, dtype=torch.float16, out=z)
    with pytest.raises(ValueError):
        asv.lm_head_logits(x, head, out=torch.zeros((N, V + 1), device=dev))
    with pytest.raises(ValueError):
        asv.lm_head_logits(x, head, out=torch.zeros((V, N), device=dev).t())
    with pytest.raises(ValueError):
        asv.lm_head_logits(x, head, workspace=torch.zeros(8, dtype=torch.uint8, device=dev))
    with pytest.raises(TypeError):
        asv.pack_lm_head_fp8(w, torch.zeros((3, 1), dtype=torch.uint8, device=dev))
    with pytest.raises(ValueError):
        asv.pack_lm_head_fp8(w.to(torch.float8_e4m3fn), torch.zeros((2, 1), dtype=torch.uint8, device=dev))
    args = (x, head, i(1, 2, 3, 4), i(-1, 0, 1, 2), i(0, 4), torch.zeros(1, device=dev))
    for kw in (dict(k1_tile=64), dict(noalloc=True)):
        with pytest.raises(ValueError):
            asv.verify(*args, **kw)
        with pytest.raises(ValueError):
            asv.verify(x, w, *args[2:], rules=asv.LogitRules(), **kw)
    for bad in (dict(counts=torch.zeros((1, V), device=dev)), dict(counts=i(*range(V))), dict(bias=one),
                dict(bias=torch.zeros((2, V), device=dev)), dict(allowed=i(1)), dict(repetition=one.double()),
                dict(presence=one), dict(frequency=torch.ones(1))):
        with pytest.raises((TypeError, ValueError)):
            asv.verify(*args, rules=asv.LogitRules(**bad))
        with pytest.raises((TypeError, ValueError)):
            asv.adjust_logits(z, asv.LogitRules(**bad), i(0, 4))
    with pytest.raises(ValueError):
        asv.adjust_logits(z, asv.LogitRules(), i(0, 4), parent=i(-1, 0, 1, 2))
    with pytest.raises(TypeError):
        asv.adjust_logits(z, asv.LogitRules(), out=z.half())
    with pytest.raises(asv.AsvError):                                   # overlaps, and is not the input
        buf = torch.zeros((N + 1) * V, device=dev)
        asv.adjust_logits(buf[:N * V].view(N, V), asv.LogitRules(), out=buf[V:].view(N, V))
    with pytest.raises(TypeError):
        asv.token_counts(i(1, 2).long(), i(0, 2), V)
    with pytest.raises(ValueError):
        asv.token_counts(i(1, 2), i(0, 2), V, counts=i(1, 2))
    with pytest.raises(ValueError):
        asv.token_counts(i(1, 2), i(0, 2), V, prompt_len=i(1, 2))


def test_nothing_to_do(asv, dev):
    """No rows, no requests, no tokens."""
    import torch
    V, H = 300, 64
    head = asv.quantize_lm_head(torch.zeros((V, H), dtype=torch.bfloat16, device=dev))
    none = torch.zeros((0, H), dtype=torch.bfloat16, device=dev)
    assert asv.lm_head_logits(none, head).shape == (0, V)
    assert asv.adjust_logits(torch.zeros((0, V), device=dev), asv.LogitRules()).shape == (0, V)
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev)       # noqa: E731
    c, st = asv.token_counts(i(), i(0), V)
    assert c.shape == (0, V) and st.shape == (0,)
    c, st = asv.token_counts(i(), i(0, 0, 0), V)
    assert not c.any() and not st.any()
