"""Rotation: components behind the pairs pass as they are, whatever lies beside them."""
import pytest
import torch

import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, F32 = cngp.F16, cngp.F32


# pairs that end inside a 16-byte piece (next), on one (halves), heads by single values, no pairs at all
@pytest.mark.parametrize("D,pairs,nxt", [(36, (3, 3, 3), True), (24, (2, 4), True), (64, (8, 8), False), (7, (2,), False), (7, (2,), True), (16, (0,), False), (512, (0, 8), False)])
@pytest.mark.parametrize("io", [F16, F32])
def test_components_behind_the_pairs_next_to_ones_that_are_not_finite(D, pairs, nxt, io):
    N, H, K = 70, 3, 2
    g = torch.Generator().manual_seed(D)
    dtype = torch.float16 if io == F16 else torch.float32
    cfg = cngp.RotateConfig(H, K, D, pairs, io, flags=cngp.ROTATE_NEXT if nxt else 0)
    turned = 2 * sum(pairs)
    position, omega = torch.rand(N, len(pairs), generator=g).to(DEV), torch.ones(sum(pairs), device=DEV)
    for odd in (float("inf"), float("-inf"), float("nan")):
        x = [torch.randn(N, h, D, generator=g).to(dtype) for h in (H, K)]
        for t in x:
            t[..., turned:][torch.rand(t[..., turned:].shape, generator=g) < 0.3] = odd
        q, k = (t.to(DEV) for t in x)
        args = (position, omega) if sum(pairs) else (None, None)
        for out in (cngp.rotate_fwd(cfg, q, k, *args), cngp.rotate_bwd(cfg, None, None, *args, q, k)[:2]):
            for a, b in zip(out, (q, k)):
                assert torch.equal(torch.nan_to_num(a[..., turned:], 1.0, 2.0, 3.0), torch.nan_to_num(b[..., turned:], 1.0, 2.0, 3.0))
                assert bool(torch.isfinite(a[..., :turned]).all())
