"""The 8-bit LM head on more rows than one launch has workgroups of 256 threads for."""

import pytest

pytestmark = pytest.mark.gpu


def test_more_rows_than_a_launch_has_workgroups():
    """2^24 rows and a few: 256 threads a row are 2^32. The rows around every seam and the last ones are those
    of a call on them alone, as are the records of verification."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_02897_amd as asv
    dev, N, V, H = torch.device("cuda:0"), (1 << 24) + 37, 3, 64
    g = torch.Generator(device=dev).manual_seed(1)
    x = torch.randn((N, H), device=dev, generator=g, dtype=torch.bfloat16)
    head = asv.quantize_lm_head(torch.randn((V, H), device=dev, generator=g).bfloat16())
    z = asv.lm_head_logits(x, head)
    seams = [(0, 40), ((1 << 23) - 20, (1 << 23) + 20), ((1 << 24) - 20, N)]
    for lo, hi in seams:
        assert torch.equal(z[lo:hi], asv.lm_head_logits(x[lo:hi].contiguous(), head))
    B, per = 1024, N // 1024
    off = per * torch.arange(B + 1, dtype=torch.int32, device=dev)
    off[-1] = N
    parent = off[(torch.arange(N, device=dev) // per).clamp(max=B - 1)]     # every node under its root
    parent[off[:-1].long()] = -1
    out = asv.verify(x, head, torch.zeros(N, dtype=torch.int32, device=dev), parent, off,
                     torch.full((B,), 0.5, device=dev))
    assert not out.req_status.any() and torch.equal(out.row_max, z.max(1).values)
    assert torch.equal(out.row_argmax, z.argmax(1).int())
