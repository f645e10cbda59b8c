"""Drafted tokens taken back, inside the open block and across a block that they filled: the open rows put back as they were before
the drafts, and the tokens that stay appended again.  The cache and what its readers give are then, to the bit, those of a cache
that never had the drafts."""
import pytest
import torch

import paper_2412_06198_amd as sa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [sa.SA_CACHE_E4M3, sa.SA_CACHE_E5M2])
@pytest.mark.parametrize("b", [64, 128])
def test_drafts_taken_back(b, kind):
    N, hq, hkv, drafts = 512, 8, 2, 5
    gen = torch.Generator(device="cuda").manual_seed(b + kind)
    ses = sa.Session(hq, hkv, N, b, 64, keep=0.3)
    Q, K, V, DK, DV = (torch.randn((h, N + 2 * b, 128), generator=gen, device="cuda").bfloat16() for h in (hq, hkv, hkv, hkv, hkv))
    ses.estimate_and_index(Q[:, :N].contiguous(), K[:, :N].contiguous())
    for at in range(b - drafts - 1, b + 1):   # tokens in the block before the drafts
        for stay in range(drafts + 1):        # of the drafts
            print(f"case take back b={b} kind={kind} at={at} stay={stay}", flush=True)
            pos = N + at
            plain, c = ses.cache(N + 2 * b, kind), ses.cache(N + 2 * b, kind)
            for x in (plain, c):
                for t in x.tensors:
                    t.view(torch.uint8).fill_(0x7F)
                ses.append(x, K[:, :pos], V[:, :pos], 0)
            kept = c.k_open.clone(), c.v_open.clone()
            dk, dv = DK[:, :drafts].clone(), DV[:, :drafts].clone()
            dk[:, :stay], dv[:, :stay] = K[:, pos:pos + stay], V[:, pos:pos + stay]
            ses.append(c, dk, dv, pos)
            o = torch.empty((hq, drafts, 128), dtype=torch.bfloat16, device="cuda")
            ses.attend(c, Q[:, pos:pos + drafts], pos, o)
            c.k_open.copy_(kept[0])
            c.v_open.copy_(kept[1])
            ses.append(c, K[:, pos:pos + stay], V[:, pos:pos + stay], pos)
            end = pos + stay
            ses.append(plain, K[:, pos:end], V[:, pos:end], pos)
            for step in range(2):             # and the generation goes on
                for x in (plain, c):
                    ses.append(x, K[:, end:end + 1], V[:, end:end + 1], end)
                end += 1
                full, rest = end // b * b, end % b
                for x, y in zip(c.tensors[:4], plain.tensors[:4]):
                    n = full if x.dtype == torch.uint8 else full // b
                    assert torch.equal(x[:, :n], y[:, :n])
                assert torch.equal(c.k_open[:, :rest], plain.k_open[:, :rest]) and torch.equal(c.v_open[:, :rest], plain.v_open[:, :rest])
                q = Q[:, end - 1:end].contiguous()
                got, want = torch.empty_like(q), torch.empty_like(q)
                ses.attend(c, q, end - 1, got)
                ses.attend(plain, q, end - 1, want)
                assert torch.equal(got, want)
                ses.decode_cached(c, q.view(hq, 128), end - 1, got.view(hq, 128))
                ses.decode_cached(plain, q.view(hq, 128), end - 1, want.view(hq, 128))
                assert torch.equal(got, want)
