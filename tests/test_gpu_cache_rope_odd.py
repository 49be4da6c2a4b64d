"""sp_qk_norm_rope beside elements that are not finite: one of them reaches its pair's partner and, with a norm, its head's mean, and
nothing else."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

HALF_BF16 = 2.0 ** -8     # half a step of bf16, relative


def _bits(t):
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy()


# tokens from 4096 on with rows that do not fill a workgroup: four tokens to a workgroup
@pytest.mark.parametrize("tokens,hq,hk,d,rotary", [
    (9, 4, 2, 128, 0), (9, 4, 2, 64, 0), (33, 3, 1, 128, 8), (33, 6, 2, 128, 64), (20, 4, 4, 64, 32), (17, 2, 1, 64, 56), (17, 2, 1, 128, 120),
    (4099, 3, 3, 64, 24), (4097, 2, 1, 128, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_an_element_that_is_not_finite_touches_its_pair_alone(tokens, hq, hk, d, rotary, interleaved, norm):
    """Element by element against 64 bits; what is neither rotated nor normed comes out bit for bit, signs of zeros among it.
    Tolerance of the finite ones: half a bf16 step of the result, and 2^-16 of the pair for the 32-bit arithmetic."""
    import torch
    import paper_2505_19578_amd as sp
    from oracle import cache as oracle
    torch.manual_seed(tokens + d + rotary)
    rng = np.random.default_rng(tokens + d + rotary)
    x = torch.randn(tokens, hq + 2 * hk, d) * 3
    odd = [float("nan"), float("inf"), -float("inf"), -0.0, 0.0]
    for n, (t, h) in enumerate((t, h) for t in range(min(tokens, 33)) for h in range(hq + 2 * hk)):
        for e in rng.choice(d, n % 3, replace=False):       # none, one or two in a head
            x[t, h, int(e)] = odd[int(rng.integers(0, 5))]
    qkv = x.to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    w = [(torch.rand(d) + 0.5).to(torch.bfloat16).cuda() if norm else None for _ in range(2)]
    inv = (10000.0 ** (-torch.arange(0, max(rotary, 2), 2, dtype=torch.float64) / max(rotary, 1))).float().cuda()
    pos = torch.randint(1, 1 << 17, (tokens,), dtype=torch.int32).cuda()
    q_out, k_out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    page = 32
    kc, vc = (torch.full((tokens // page + 1, page, hk, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots = torch.randperm(tokens).to(torch.int32).cuda()
    shape = sp.rope_shape_of(q, k, v, q_out, k_out, rotary, interleaved, 1e-5)
    print(f"[rope] {tokens} tokens, {rotary} of {d}, interleaved {interleaved}, norm {norm}", flush=True)
    sp.sp_qk_norm_rope(shape, q, k, v, w[0], w[1], inv, pos, q_out, k_out, sp.cache_shape_of(kc), kc, vc, slots)
    torch.cuda.synchronize()
    for src, out, weight in ((q, q_out, w[0]), (k, k_out, w[1])):
        with np.errstate(invalid="ignore"):
            want, size = oracle.norm_rope(src.float().cpu().numpy(), None if weight is None else weight.float().cpu().numpy(), 1e-5,
                                          pos.cpu().numpy(), inv[:rotary // 2].cpu().numpy(), rotary, interleaved)
            got = out.float().cpu().numpy().astype(np.float64)
            near = np.abs(got - want) <= HALF_BF16 * np.abs(want) + 2.0 ** -16 * size + 1e-30
        same = np.where(np.isfinite(want), near, (got == want) | (np.isnan(got) & np.isnan(want)))
        assert same.all(), (np.argwhere(~same)[:5], got[~same][:5], want[~same][:5])
        if not norm:
            a, b = _bits(src[..., rotary:]), _bits(out[..., rotary:])
            assert ((a == b) | (np.isnan(src[..., rotary:].float().cpu().numpy()) & np.isnan(got[..., rotary:]))).all()
    flat = slots.long()
    for cache, rows in ((kc, k_out), (vc, v)):
        assert np.array_equal(_bits(cache.view(-1, hk, d)[flat]), _bits(rows))
