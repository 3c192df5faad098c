"""Plain float64 forms of the 8-bit LM head and of the sampling rules, for their tests: written from
the definitions in include/asv.h, node by node."""

from __future__ import annotations

import numpy as np

import oracle

BLOCK = 128
PROMPT = 1 << 30

# the 256 values of e4m3 (OCP): sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff NaN
E4M3 = np.array([np.nan if (c & 127) == 127 else
                 (-1) ** (c >> 7) * ((c & 7) / 8 * 2.0 ** -6 if (c >> 3 & 15) == 0 else
                                     (1 + (c & 7) / 8) * 2.0 ** ((c >> 3 & 15) - 7))
                 for c in range(256)])
_POS = E4M3[:127]                      # the codes of the values >= 0, ascending


def e4m3_codes(x: np.ndarray) -> np.ndarray:
    """The nearest code of every |x| <= 448, ties to the even code."""
    a = np.abs(x)
    hi = np.searchsorted(_POS, a).clip(0, 126)            # least value >= a
    lo = np.maximum(hi - 1, 0)
    up, down = _POS[hi] - a, a - _POS[lo]
    c = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    c = np.where(_POS[hi] == a, hi, c)
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def block_scale(x: np.ndarray) -> int:
    """The E8M0 byte of a block: the least k >= -126 with |x| <= 448 * 2^k, plus 127."""
    a = np.abs(x).max() if x.size else 0.0
    if not np.isfinite(a):
        return 255
    k = -126
    while a > 448.0 * 2.0 ** k:
        k += 1
    return k + 127


def quantise(x: np.ndarray, rows: int):
    """(codes, scales [ceil(R / rows)][ceil(H / 128)], values) of x float64 [R][H] in blocks of
    `rows` x 128."""
    R, H = x.shape
    codes, value = np.zeros((R, H), dtype=np.uint8), np.empty((R, H))
    scale = np.zeros((-(-R // rows), -(-H // BLOCK)), dtype=np.uint8)
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            at = np.s_[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK]
            s = block_scale(x[at])
            scale[i, j] = s
            if s == 255:
                value[at] = np.nan
                continue
            step = 2.0 ** (s - 127)
            codes[at] = e4m3_codes(x[at] / step)
            value[at] = E4M3[codes[at]] * step
    return codes, scale, value


def path_tokens(n: int, parent, draft_tok) -> list:
    out = []
    while parent[n] >= 0:
        out.append(int(draft_tok[n]))
        n = int(parent[n])
    return out


def ruled(z: np.ndarray, rules: dict, off=None, parent=None, draft_tok=None) -> np.ndarray:
    """The rules on float64 logits z [N][V]; rules as numpy arrays by LogitRules' names."""
    N, V = z.shape
    off = np.arange(N + 1) if off is None else off
    out = z.copy()

    def of(name, b, default):
        return default if rules.get(name) is None else float(rules[name][b])

    for b in range(len(off) - 1):
        table = rules.get("counts")
        base = np.zeros(V, dtype=np.int64) if table is None else table[b].astype(np.int64)
        rep, pres, freq = of("repetition", b, 1.0), of("presence", b, 0.0), of("frequency", b, 0.0)
        for n in range(int(off[b]), int(off[b + 1])):
            g = base % PROMPT
            seen = base > 0
            if parent is not None:
                for t in path_tokens(n, parent, draft_tok):
                    if 0 <= t < V:
                        g[t] += 1
                        seen[t] = True
            row = out[n]
            row = np.where(seen, np.where(row > 0, row / rep, row * rep), row)
            row = np.where(g > 0, row - (pres + freq * g), row)
            if rules.get("bias") is not None:
                bias = rules["bias"]
                row = row + (bias if bias.ndim == 1 else bias[b]).astype(np.float64)
            if rules.get("allowed") is not None:
                v = np.arange(V)
                on = (rules["allowed"][n].view(np.uint32)[v // 32] >> (v % 32).astype(np.uint32)) & 1
                row = np.where(on == 1, row, -np.inf)
            out[n] = row
    return out


def verify(z: np.ndarray, w, tau, params=None, ban: bool = True, state=None) -> dict:
    """Every output of one verification step on given logits: the oracle's row statistics, margin
    rule and walk. With `ban`, a drafted token of -inf is never accepted and a row without
    any finite logit has the argmax -1."""
    params = params or oracle.Params()
    with np.errstate(invalid="ignore", divide="ignore"):
        M, a, L, gap = oracle.row_stats(z)
        empty = ~np.isfinite(M)
        L = np.where(empty, -np.inf, L)
        a = np.where(empty, -1, a)
        gap = np.where(empty, np.inf, gap)
        N = len(w.parent)
        g = np.zeros(N)
        for c in range(N):
            if w.parent[c] >= 0:
                g[c] = z[w.parent[c], w.draft_tok[c]]
        tau_node = np.empty(N)
        for b in range(w.B):
            tau_node[w.req_offsets[b]:w.req_offsets[b + 1]] = float(np.float32(tau[b]))
        acc = oracle.accept_flags(g, M, a, w.parent, w.draft_tok, tau_node, params.temperature)
        if ban:
            acc &= (np.asarray(w.parent) < 0) | (g > -np.inf)
        out = dict(row_max=M, row_lse=L, row_argmax=a, row_gap=gap, drafted_logit=g, accept=acc,
                   tau_node=tau_node, accepted_len=np.zeros(w.B, dtype=np.int64),
                   bonus_token=np.zeros(w.B, dtype=np.int64),
                   accepted_path=np.full(N, -1, dtype=np.int64),
                   band_at=np.full(w.B, -1, dtype=np.int64), temperature=params.temperature)
        for b in range(w.B):
            lo, hi = int(w.req_offsets[b]), int(w.req_offsets[b + 1])
            path, n, bonus = oracle.walk(lo, hi, w.parent, w.draft_tok, g, acc, a,
                                         params.max_promotions)
            out["accepted_len"][b], out["bonus_token"][b] = n, bonus
            out["accepted_path"][lo:lo + n] = path
    return out
