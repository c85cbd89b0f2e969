"""Operands whose rows lie further than 2^32 bytes apart: the far rows get what a call on them alone gives, bit for bit where one row's
work does not depend on the others, else within the tolerance of its own tests."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def c2r():
    from paper_2504_01337_amd import c2r as m
    m.lib()
    return m


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_norm(c2r):
    T, d = 300000, 8192                                              # 4.9 GB
    x = torch.empty((T, d), dtype=torch.bfloat16, device="cuda").normal_(generator=_gen(1))
    y, _, y8, c = c2r.add_rms_norm(x, bits8=True)
    for rows in (slice(0, 5), slice(262140, 262150), slice(T - 5, T)):
        ref = c2r.add_rms_norm(x[rows], bits8=True)
        assert torch.equal(y[rows], ref[0]) or (y[rows].float() - ref[0].float()).abs().max() <= 2.0 ** -7 * ref[0].float().abs().max()
        assert torch.equal(y8[rows].view(torch.uint8), ref[2].view(torch.uint8)) and torch.equal(c[rows], ref[3])


def test_logprobs(c2r):
    T, V = 18000, 128256                                             # 4.6 GB
    l = torch.empty((T, V), dtype=torch.bfloat16, device="cuda").normal_(generator=_gen(2))
    tok = torch.randint(0, V, (T, 2), generator=_gen(3), dtype=torch.int32, device="cuda")
    lp, ent, top, top_lp = c2r.token_logprobs(l, tok, 5)
    for rows in (slice(0, 3), slice(16740, 16746), slice(T - 3, T)):  # (row 16744 begins before 2^32 and ends behind it)
        ref = c2r.token_logprobs(l[rows], tok[rows].contiguous(), 5)
        assert torch.equal(top[rows], ref[2])
        # sums of V / 256 + 64 terms in another order on either side, against distances of up to 12: 2 * 2^-24 * (4 * 12 + 600) < 2^-13
        for a, b in ((lp[rows], ref[0]), (ent[rows], ref[1]), (top_lp[rows], ref[3])):
            assert (a - b).abs().max() <= 2.0 ** -13 * 4


def test_adapters(c2r):
    T, d_in, d_out, n = 370000, 64, 6144, 3                          # y: 4.5 GB
    y = torch.empty((T, d_out), dtype=torch.bfloat16, device="cuda").normal_(generator=_gen(4))
    x = torch.empty((T, d_in), dtype=torch.bfloat16, device="cuda").normal_(generator=_gen(5))
    A, B = (torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(generator=_gen(6)) for s in ((n, 8, d_in), (n, d_out, 8)))
    ids = (torch.arange(T, dtype=torch.int32, device="cuda") // 1000 % (n + 1) - 1).contiguous()
    rows = [slice(0, 40), slice(349510, 349540), slice(T - 40, T)]
    keep = [y[r].clone() for r in rows]
    c2r.adapters(x, ids, A, B, y, out=y)
    for r, k in zip(rows, keep):
        ref = c2r.adapters(x[r], ids[r].contiguous(), A, B, k)
        # one rounding to bf16 on either side of sums that differ by their order: 2 * 2^-8 of the larger
        assert ((y[r].float() - ref.float()).abs() <= 2.0 ** -7 * ref.float().abs() + 2.0 ** -10).all()
