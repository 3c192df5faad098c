"""The roundings of the sampling rules on logits in memory. A quotient by the repetition is taken as the
product with its reciprocal, rounded to fp32: z1 = z (1 / rep), two roundings; the other operations round once each.

With u = 2^-24, in exact arithmetic z1 = z / rep or z rep, p = presence + frequency g, z2 = z1 - p, z3 = z2 + bias,
and errors e of what was computed: e1 <= 2 u |z1|, ep <= u |p|, e2 <= e1 + ep + u |z2|, e3 <= e2 + u |z3|; the
products of two u are covered by a factor of 1 + 2^-20. Stored in 16 bits, half a step of the result more."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

PROMPT = 1 << 30


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


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [1, 37, 4100])
def test_each_operation_rounds_once(asv, dev, dtype, V):
    import torch
    N = 40
    rng = np.random.default_rng(V)
    t = lambda a: torch.from_numpy(a).to(dev)                       # noqa: E731
    x = t((5 * rng.standard_normal((N, V))).astype(np.float32)).to(getattr(torch, dtype))
    g = np.where(rng.random((N, V)) < 0.5, rng.integers(1, 40, (N, V)), 0)
    prompt = rng.random((N, V)) < 0.3
    rep = np.exp(rng.uniform(-2, 2, N)).astype(np.float32)
    pres, freq = (rng.standard_normal(N).astype(np.float32) for _ in range(2))
    bias = (3 * rng.standard_normal((N, V))).astype(np.float32)
    got = asv.adjust_logits(x, asv.LogitRules(t((g + PROMPT * prompt).astype(np.int32)), t(rep), t(pres), t(freq),
                                              t(bias))).double().cpu().numpy()
    z = x.double().cpu().numpy()
    r, one = rep.astype(np.float64)[:, None], 1.0
    z1 = np.where((g > 0) | prompt, np.where(z > 0, z / r, z * r), z)
    p = np.where(g > 0, pres.astype(np.float64)[:, None] + freq.astype(np.float64)[:, None] * g, 0.0)
    z2 = z1 - p
    z3 = z2 + bias
    tol = (one + 2.0 ** -20) * 2.0 ** -24 * (2 * np.abs(z1) + np.abs(p) + np.abs(z2) + np.abs(z3))
    half = {"float32": 0.0, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dtype]
    tol = tol + half * (np.abs(z3) + tol) + (2.0 ** -25 if dtype == "float16" else 0.0)
    bad = np.argwhere(~(np.abs(got - z3) <= tol))
    assert len(bad) == 0, (bad[:4], got[tuple(bad[0])], z3[tuple(bad[0])])


def test_repetitions_and_their_reciprocals(asv, dev):
    """Bit for bit, over the whole range: below 2^-128 the reciprocal is infinite, and so is what a positive logit
    of a seen id becomes."""
    import torch
    reps = np.array([0.0, 1e-44, 1e-40, 2.9e-39, 3e-39, 1.2e-38, 1e-30, 0.1, 0.7, 1.0, 1.3, 3.0, 1e30, 1e38, 3.4e38,
                     np.inf], dtype=np.float32)
    rng = np.random.default_rng(4)
    V = 200
    z = np.concatenate([rng.standard_normal(V - 8), [0.0, 1e-38, -1e-38, 1e38, -1e38, 1e-3, -1e-3, 1.0]])
    z = np.tile(z.astype(np.float32), (len(reps), 1))
    t = lambda a: torch.from_numpy(a).to(dev)                       # noqa: E731
    got = asv.adjust_logits(t(z), asv.LogitRules(t(np.full(z.shape, PROMPT, np.int32)), t(reps))).cpu().numpy()
    with np.errstate(all="ignore"):
        inv = np.float32(1.0) / reps
        want = np.where(z > 0, z * inv[:, None], z * reps[:, None])
    assert want.dtype == np.float32 and np.isinf(inv[:4]).all() and np.isfinite(inv[4])
    assert np.array_equal(got, want, equal_nan=True)
