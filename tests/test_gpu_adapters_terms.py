"""The bf16 terms of X A^T in mwu_adapters_add, by numbers that need all of them.

T = X A^T is a sum of three products with 8, 8 and 8 bits of one 24-bit number, exact in fp32; B is a signed unit matrix, so Y = +-T.
An fp32 Y holds T in three terms: with the parts added up exactly (24 bits in all) Y is T; what the tensor core may lose of a running
sum, 2^-22 a step over at most rank / 16 * 3 + 2 steps of which all but two add zeros, is granted twice: 2^-21.  A third term left out
would cost 2^-17 of some T: the test looks that its numbers show that.  A bf16 Y: two terms, 2^-17, and half a step, 2^-8."""
import pytest
import torch

from test_gpu_adapters import Batch
from test_gpu_grouped import F64

pytestmark = pytest.mark.gpu


def split(t, terms):
    """The sum of the first bf16 terms of fp32 numbers."""
    s, out = t.clone(), torch.zeros_like(t, dtype=F64)
    for _ in range(terms):
        h = s.to(torch.bfloat16).float()
        out, s = out + h.to(F64), s - h
    return out


@pytest.mark.parametrize("fp32", [1, 0])
@pytest.mark.parametrize("rank", [16, 32, 64, 128, 5, 40])
@pytest.mark.parametrize("lengths", [[7, 9], [200], [33, 1, 300]], ids=str)
def test_numbers_of_24_bits(lengths, rank, fp32):
    cols, rows = 200, 2 * rank
    b = Batch(lengths, [0] * len(lengths), 1, rank, rows, cols, fp32, with_scale=False)
    g = torch.Generator(device="cuda")
    g.manual_seed(rank)
    bits = lambda lo: torch.randint(lo, 256, (rank,), generator=g, device="cuda").float()
    a0, a1, a2 = bits(128), bits(0), bits(1)
    b.A[:, :rank, :cols] = 0
    b.A[0, :rank, 3], b.A[0, :rank, 90], b.A[0, :rank, 170] = a0.to(b.A.dtype), a1.to(b.A.dtype), a2.to(b.A.dtype)
    b.X[:b.M, :cols] = 0
    sign = torch.ones(b.M, device="cuda")
    sign[::3] = -1
    for k, step in ((3, 1.0), (90, 2.0 ** -8), (170, 2.0 ** -16)):
        b.X[:b.M, k] = (sign * step).to(b.X.dtype)
    b.B[:, :rows, :rank] = 0
    eye = torch.eye(rank, device="cuda").to(b.B.dtype)
    b.B[0, :rank, :rank], b.B[0, rank:rows, :rank] = eye, -eye
    T = a0.to(F64) + a1.to(F64) * 2.0 ** -8 + a2.to(F64) * 2.0 ** -16
    assert torch.equal(T.float().to(F64), T)                # 24 bits
    Y = torch.zeros_like(b.Y0)
    b.run(None, Y)
    torch.cuda.synchronize()
    assert int(b.st.item()) == 0
    ref = sign.to(F64)[:, None] * torch.cat([T, -T])
    tol = ref.abs() * (2.0 ** -21 if fp32 else 2.0 ** -8 + 2.0 ** -17)
    assert bool(((Y[:, :rows].to(F64) - ref).abs() <= tol).all())
    if fp32:                                                # and two terms would not do
        assert bool(((split(T.float(), 2) - T).abs() > T * 2.0 ** -21).any()) and torch.equal(split(T.float(), 3), T)
