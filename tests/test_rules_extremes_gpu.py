"""Sampling rules that force or ban ids by the size of a bias or a penalty, infinite or merely huge: verification on
either weight, in the fused and the unfused finishing step, against float64.

Weights and hidden states are powers of two, so that every logit before the rules is exact and both heads hold
the same ones. A ruled logit is then z + bias rounded once to fp32 (z / rep and z * rep: twice), and the tests take
their float64 values from the fp32 ones that the rules give.

Tolerance of row_lse = m + ln(sum exp(z - m)): 2^-24 (4 |m| + 4 |lse| + 256). The exponent is
z log2(e) - m log2(e), whose second product is rounded: 2^-24 |m| of the sum, a share of |m| once more for
the constant's own rounding where z and m differ. Each exponential is one unit of 2^-23 off and its argument
2^-24 of itself (x e^-x < 1/2), and a row's sum goes through fewer than 100 additions of positive terms: together
below 2^-24 * 256 with the logarithm's own unit. The last addition rounds to 2^-24 |lse|, the
product before it to less."""

import numpy as np
import pytest

import rules_oracle as ro

pytestmark = pytest.mark.gpu

FMAX = float(np.finfo(np.float32).max)


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


class Step:
    """B requests of n nodes each (chains) on a V-id head, with exact logits z float64 [N][V]."""

    def __init__(self, dev, B, n, V, seed):
        import torch
        H = 64
        self.rng = np.random.default_rng([seed, B, n, V])
        pick = lambda *s: 2.0 ** self.rng.integers(-2, 1, s) * self.rng.choice([-1.0, 1.0], s)  # noqa: E731
        self.B, self.N, self.V, self.dev = B, B * n, V, dev
        x, w = pick(self.N, H), pick(V, H)
        self.z = x @ w.T
        self.x, self.w = (torch.from_numpy(a).to(dev).bfloat16() for a in (x, w))
        self.parent = np.where(np.arange(self.N) % n == 0, -1, np.arange(self.N) - 1).astype(np.int32)
        self.off = (n * np.arange(B + 1)).astype(np.int32)
        self.tok = self.rng.integers(0, V, self.N).astype(np.int32)
        self.tau = self.rng.choice([0.0, 0.3, 1.0], B).astype(np.float32)

    def run(self, asv, head, rules):
        import torch
        w = {"row": lambda: self.w, "packed": lambda: asv.pack_lm_head(self.w),
             "fp8": lambda: asv.quantize_lm_head(self.w)}[head]()
        out = asv.verify(self.x, w, *(_t(a, self.dev) for a in (self.tok, self.parent, self.off, self.tau)),
                         rules=asv.LogitRules(**{k: _t(v, self.dev) for k, v in rules.items()}))
        torch.cuda.synchronize()
        return {f: getattr(out, f).cpu().numpy() for f in out._fields if f != "draft_conf"}

    def check(self, asv, head, rules):
        """Every output against the definition, on the fp32 ruled logits."""
        with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
            zr = ro.ruled(self.z, rules, self.off, self.parent, self.tok).astype(np.float32).astype(np.float64)
            assert not np.isnan(zr).any()
            m, arg = zr.max(1), zr.argmax(1)
            part = np.where(zr == m[:, None], 0.0, zr - m[:, None])
            lse = m + np.log(np.exp(part).sum(1))
            up = np.maximum(self.parent, 0)
            g = zr[up, self.tok]
            tau = np.repeat(self.tau, np.diff(self.off)).astype(np.float64)
            ok = (self.tok == arg[up]) | (tau == 0) | (g == m[up]) | (g - m[up] >= np.log(tau))
        ok = (self.parent < 0) | (ok & (g > -np.inf))
        got = self.run(asv, head, rules)
        assert np.array_equal(got["row_max"], m) and np.array_equal(got["row_argmax"], arg)
        kid = self.parent >= 0
        assert np.array_equal(got["drafted_logit"][kid], g[kid])
        big = np.isinf(m)
        assert np.array_equal(got["row_lse"][big], m[big]), got["row_lse"][big]
        off = np.abs(got["row_lse"][~big] - lse[~big])
        tol = 2.0 ** -24 * (4 * np.abs(m[~big]) + 4 * np.abs(lse[~big]) + 256)
        assert np.all(off <= tol), (got["row_lse"][~big][~(off <= tol)][:4], lse[~big][~(off <= tol)][:4])
        assert np.array_equal(got["accept"], ok) and not got["req_status"].any()
        for b, lo in enumerate(self.off[:-1]):          # chains: as far as every node is accepted
            n = 0
            while lo + n + 1 < self.off[b + 1] and ok[lo + n + 1]:
                n += 1
            assert got["accepted_len"][b] == n and got["bonus_token"][b] == arg[lo + n]


# one row tile and several, cut ids, and more requests than the fused finishing step takes
STEPS = [(2, 9, 300), (4, 15, 2001), (10, 7, 3000), (5, 60, 1300), (1100, 2, 260)]
HEADS = ["row", "packed", "fp8"]


@pytest.mark.parametrize("B,n,V", STEPS)
@pytest.mark.parametrize("head", HEADS)
def test_infinite_ruled_logits(asv, dev, head, B, n, V):
    """A bias of +inf forces an id: of one such id, of two and of many, a repetition of 0 forces every seen id
    of a positive logit. Forced ids are the row's maximum, so drafted ones are accepted."""
    s = Step(dev, B, n, V, 1)
    bias = s.rng.standard_normal((B, V)).astype(np.float32)
    bias[0, V // 2] = np.inf
    s.tok[1] = V // 2
    bias[-1, [3, V - 1]] = np.inf
    s.tok[-n + 1] = V - 1                   # the second of two
    if B > 2:
        bias[1, s.rng.random(V) < 0.5] = np.inf
        bias[2, s.rng.random(V) < 0.5] = -np.inf
        bias[2, 7] = np.inf
    s.check(asv, head, dict(bias=bias))
    counts = (s.rng.random((B, V)) < 0.3).astype(np.int32)
    rep = np.ones(B, np.float32)
    rep[::2] = 0.0
    s.check(asv, head, dict(counts=counts, repetition=rep))


@pytest.mark.parametrize("B,n,V", STEPS)
@pytest.mark.parametrize("head", HEADS)
@pytest.mark.parametrize("size", [1e6, 1e9, 1e10, 1e30, FMAX])
def test_huge_finite_biases(asv, dev, head, size, B, n, V):
    """Ids banned and forced by a bias that is finite: bans of every id of whole slabs, of all ids of a row but one
    and of all of them, and forced ids that leave every other logit behind."""
    s = Step(dev, B, n, V, 2)
    v = np.arange(V)
    bias = np.zeros((B, V), np.float32)
    bias[0] = np.where(v // 64 % 2 == 0, -size, 0)
    bias[1] = np.where(v == V - 2, 0, -size)
    if B > 2:
        bias[2] = -size
        bias[3, s.rng.random(V) < 0.4] = size
        bias[3, s.rng.random(V) < 0.4] = -size
    if B > 4:
        bias[4, V // 3] = size
    # as many requests as there are, with these rules in turn
    for b in range(5, B):
        bias[b] = bias[b % 5]
    s.check(asv, head, dict(bias=bias))
