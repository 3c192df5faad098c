"""Every tile family and tail of the 8-bit LM head over many K stages: more of them than its ring has slots, and
hidden sizes past 512, where the scales of a row of blocks take more than one word. Logits of sampled ids
against float64: whole blocks of 128 around the seams between main slabs and tail, the first and the last
ones and some at random. The records of verification agree with the logits bit for bit, also where another
family computes them. Tolerance as in test_fp8_head_gpu."""

import numpy as np
import pytest

import rules_oracle as ro
from test_fp8_head_gpu import _check_logits

pytestmark = pytest.mark.gpu

# (rows, ids): on 256 CUs 64-id tiles; 128-id ones, alone and with a tail of 64; 256-id ones alone and with tails of 64
# and 128; 128 rows with tails of 64 and 128 and those alone; 192 rows; 256 rows, and their tail alone; two
# families in two launches
SHAPES = [(7, 16000), (60, 20001), (64, 50001), (60, 40003), (33, 70001), (9, 90001), (60, 128256), (4, 140001),
          (57, 151936), (5, 168003), (90, 75003), (100, 48003), (100, 14001), (100, 30000), (190, 40003),
          (190, 16003), (256, 70003), (333, 40003), (768, 66000)]


@pytest.mark.parametrize("N,V", SHAPES)
@pytest.mark.parametrize("H", [320, 576, 1088])
def test_many_stages(N, V, H):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_02897_amd as asv
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(N * V + H)
    rng = np.random.default_rng([N, V, H])
    w = torch.randn((V, H), device=dev, generator=g) * 2.0 ** torch.randint(-6, 0, (V, 1), device=dev, generator=g)
    # every block of a row and of 128 ids at a size of its own, so that a wrong scale shows
    size = 2.0 ** torch.randint(-4, 5, (-(-V // 128), -(-H // 128)), device=dev, generator=g)
    w *= size.repeat_interleave(128, 0)[:V].repeat_interleave(128, 1)[:, :H]
    x = torch.randn((N, H), device=dev, generator=g)
    x *= (2.0 ** torch.randint(-4, 5, (N, -(-H // 128)), device=dev, generator=g)).repeat_interleave(128, 1)[:, :H]
    w, x = w.bfloat16(), x.bfloat16()
    head = asv.quantize_lm_head(w)
    z = asv.lm_head_logits(x, head)

    last = -(-V // 128) - 1
    seams = [k * 256 * t // 128 for t in (64, 128, 256) for k in range(1, 5)]
    near = {0, 1, last - 1, last} | {s + d for s in seams for d in (-1, 0)} | set(rng.integers(0, last, 6).tolist())
    blocks = sorted(b for b in near if 0 <= b <= last)
    host = lambda t: t.double().cpu().numpy()            # noqa: E731
    xq = ro.quantise(host(x), 1)[2]
    for b in blocks:
        ids = slice(128 * b, min(128 * b + 128, V))
        _check_logits(host(z[:, ids]), xq, ro.quantise(host(w[ids]), 128)[2], "float32")

    parent = torch.arange(-1, N - 1, dtype=torch.int32, device=dev)
    tok = torch.randint(0, V, (N,), dtype=torch.int32, device=dev, generator=g)
    out = asv.verify(x, head, tok, parent, torch.tensor([0, N], dtype=torch.int32, device=dev),
                     torch.full((1,), 0.3, device=dev))
    top = z.max(1).values
    assert not out.req_status.any() and torch.equal(out.row_max, top)
    assert torch.equal(out.row_argmax, (z == top[:, None]).int().argmax(1).int())
    assert torch.equal(out.drafted_logit[1:], z[:-1].gather(1, tok[1:, None].long())[:, 0])

