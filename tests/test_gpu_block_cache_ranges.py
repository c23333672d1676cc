"""Attention of the block cache with queries and scales at the ends of their ranges, against
float64 on the CPU: |error| <= 2^-8 (A + |o|) + 2^-11 A + n 2^-25 max|v| with A = sum_j p_j |v_j|
(a probability is rounded to fp16 or bf16, the output to bf16; the logits here are sums of a
few dozen exact terms of equal size: their error is under 2^-12)."""
import pytest

pytestmark = pytest.mark.gpu
D, N = 128, 64


def _run(q, k, v, scale):
    """One step over tokens k, v [n, D] (the last one new); checked against the cache's values."""
    import torch
    import paper_2608_05326_amd as qv
    n, G = k.shape[0] - 1, q.shape[0]
    k, v = k.bfloat16(), v.bfloat16()
    q = q.bfloat16()
    bc = qv.BlockCache(qv.BlockConfig(1, G, 1, n + 1, softmax_scale=scale))
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    kd, vd = k[:, None].cuda(), v[:, None].cuda()
    bc.store(0, kd[:n], vd[:n], cu)
    bc.lens = torch.tensor([n], dtype=torch.int32)
    out = torch.zeros(1, G, D, dtype=torch.bfloat16, device="cuda")
    bc.attend(0, q[None].cuda(), kd[n:].contiguous(), vd[n:].contiguous(), out)
    got = out[0].double().cpu()
    full = n // N
    kk, vv = k.double(), v.double()
    for b in range(full):
        kk[b * N:(b + 1) * N] = bc.k_codes[0, b, 0].cpu().double() * bc.k_scale[0, b, 0].cpu().double()
        vv[b * N:(b + 1) * N] = bc.v_codes[0, b, 0].cpu().double().T * bc.v_scale[0, b, 0].cpu().double()
    p = torch.softmax((q.double() @ kk.T) * (scale or D ** -0.5), dim=1)
    o, A = p @ vv, p @ vv.abs()
    tol = 2.0 ** -8 * (A + o.abs()) + 2.0 ** -11 * A + (n + 1) * 2.0 ** -25 * vv.abs().max()
    err = (got - o).abs()
    assert bool((err <= tol).all()), (err / tol).max().item()
    return A


def _aligned(n, seed):
    """Signs [D] and keys [n, D] of ones whose products with them spread from -D to D."""
    import torch
    g = torch.Generator().manual_seed(seed)
    s = torch.randn(D, generator=g).sign()
    share = torch.rand(n, 1, generator=g)
    return s, torch.where(torch.rand(n, D, generator=g) < share, s, -s)


@pytest.mark.parametrize("n", [320, 700])
@pytest.mark.parametrize("scale,qe,ke", [(0.0171, -126, 127), (0.0171, -133, 127), (2.0 ** -64, 0, 60),
                                         (0.0, -20, 20), (0.0171, 127, -126), (0.0, -126, 126)])
def test_smallest_queries(scale, qe, ke, n):
    """Queries down to 2^-126 (2^-133: the smallest there is) beside keys up to 2^127: logits of a few units."""
    import torch
    s, k = _aligned(n + 1, n)
    v = torch.randn(n + 1, D, generator=torch.Generator().manual_seed(1))
    _run(torch.stack([s, -s, s * 0.5 if qe > -126 else s]).double().mul(2.0 ** qe), k.double().mul(2.0 ** ke), v, scale)


def test_zero_logits_of_the_largest_values():
    """Query and keys of 2^127 in different channels: every logit is zero, whatever the scales."""
    import torch
    q, k = torch.zeros(1, D, dtype=torch.float64), torch.zeros(321, D, dtype=torch.float64)
    q[0, 0] = k[:, 5] = 2.0 ** 127
    v = torch.randn(321, D, generator=torch.Generator().manual_seed(2))
    _run(q, k, v, 0.0)
