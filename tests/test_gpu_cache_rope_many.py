"""sp_qk_norm_rope of more tokens than one launch takes (a grid holds fewer than 2^32 threads)."""
import pytest

pytestmark = pytest.mark.gpu


# one token to a workgroup (16 rows of 128 fill it) and four
@pytest.mark.parametrize("tokens,hq,d", [(2 ** 24 + 37, 15, 128), (2 ** 26 + 5, 1, 64)])
def test_tokens_of_several_launches(tokens, hq, d):
    """A rotation by position 0 and no norm: every key row comes out as it went in; tokens at the borders of powers of two have
    positions, and come out as in a call of themselves alone."""
    import torch
    import paper_2505_19578_amd as sp
    torch.manual_seed(1)
    k = torch.randn(tokens, 1, d, device="cuda", dtype=torch.bfloat16)
    # the query rows of neighbouring tokens are the same memory, all of one value, so that many of them take little of it
    q, q_out = (torch.full((tokens + hq - 1, d), x, device="cuda", dtype=torch.bfloat16).as_strided((tokens, hq, d), (d, d, 1)) for x in (3.0, 7.0))
    k_out = torch.full_like(k, 9.0)
    pos = torch.zeros(tokens, dtype=torch.int32, device="cuda")
    inv = torch.tensor([1.0, 0.5, 0.25, 0.125], device="cuda")
    edges = [t for n in range(20, 27) for t in (2 ** n - 1, 2 ** n, 2 ** n + 1) if t < tokens] + [0, 1, tokens - 2, tokens - 1]
    at = torch.tensor(sorted(set(edges)), device="cuda")
    if hq == 1:
        pos[at] = at.to(torch.int32) * 31 + 7
    else:           # (query rows overlap: only the keys may be told apart, so queries stay at position 0 by a rotation of 0)
        inv = torch.zeros(4, device="cuda")
    print(f"[rope] {tokens} tokens", flush=True)
    shape = sp.rope_shape_of(q, k, None, q_out, k_out, 8)
    sp.sp_qk_norm_rope(shape, q, k, None, None, None, inv, pos, q_out, k_out)
    torch.cuda.synchronize()
    few_q, few_k = q[at].contiguous(), k[at].contiguous()
    out_q, out_k = torch.empty_like(few_q), torch.empty_like(few_k)
    sp.sp_qk_norm_rope(sp.rope_shape_of(few_q, few_k, None, out_q, out_k, 8), few_q, few_k, None, None, None, inv, pos[at].contiguous(), out_q, out_k)
    assert torch.equal(k_out[at], out_k) and torch.equal(q_out[at], out_q)
    if hq == 1:
        assert not torch.equal(out_k, few_k)
    k_out[at], q_out[at] = few_k, few_q
    assert torch.equal(k_out, k)
    assert (q_out[:, 0] == 3).all() and (q_out[-1] == 3).all()
