"""Gradient of the token log probabilities at the ends of its range: large upstream gradients over masked entries, targets that are masked,
targets outside the vocabulary in rows of extreme magnitudes, and rows far from zero.

Masked entries: p = 0, so the gradient is 0 exactly, however large the upstream gradients are; the other entries have the tolerance
of test_gpu_ops_logprobs.check_backward.  Shifted rows are compared end to end, with the row's own float64 lse: the kernel's lse is off
by 2e-5 plus one rounding to fp32, half an ulp, which enters the exponent of every p; rows of |lse| >= 1024 take their sum anew and do
not have the half ulp."""
import math

import pytest
import torch

import ops_reference as R
from paper_2502_11034_b200 import logprobs
from test_gpu_ops_logprobs import DT, NINF, check_backward, strided

pytestmark = pytest.mark.gpu


def masked_rows(vocab, dtype, shift, gen):
    """Logits with masks of several kinds, targets that are not masked, and the mask."""
    lowest = torch.finfo(dtype).min
    z, _ = strided(6, vocab, dtype, vocab + 3, shift, gen)
    hidden = torch.zeros(6, vocab, dtype=torch.bool, device="cuda")
    hidden[0, ::3] = True
    hidden[1, ::3] = True
    hidden[2, vocab // 2:] = True
    hidden[3, :9] = hidden[3, -9:] = True                      # the row's unaligned ends
    hidden[4] = True
    hidden[4, 11] = False
    hidden[5, 1::2] = True
    for r, value in enumerate((NINF, lowest, lowest, NINF, NINF, -1e30)):
        z[r][hidden[r]] = value
    t = torch.tensor([1, 1, 2, 12, 11, 2], device="cuda")
    return z, t, hidden


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,shift", [(40, 0), (40, 1), (3001, 0), (3001, 3), (20011, 1)])
@pytest.mark.parametrize("c", [3.5, 4.0, 100.0, -1e4, 1e6])
def test_masked_entries_get_zero_whatever_flows_into_the_entropy(dtype, vocab, shift, c):
    gen = torch.Generator("cuda").manual_seed(vocab + shift)
    z, t, hidden = masked_rows(vocab, DT[dtype], shift, gen)
    r = logprobs.token_logprobs(z, t)
    a, b = torch.randn(6, device="cuda", generator=gen), torch.randn(6, device="cuda", generator=gen)
    cv = torch.full((6,), c, device="cuda")
    for out_shift in (shift, shift + 1):                       # lying like the logits, and not
        out, _ = strided(6, vocab, DT[dtype], vocab + 3, out_shift, gen)
        out.fill_(7.0)
        logprobs.token_logprobs_backward(z, t, r.lse, r.entropy, a, b, cv, out=out)
        assert (out[hidden] == 0).all()
        check_backward(z, t, r.lse, r.entropy, a, b, cv, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [50, 9001])
def test_target_outside_the_vocabulary_in_rows_of_extreme_magnitude(dtype, vocab):
    """The row is NaN throughout, also where p is 0."""
    gen = torch.Generator("cuda").manual_seed(vocab)
    z = (torch.randn(5, vocab, device="cuda", generator=gen) * 3 + 4096).to(DT[dtype])
    z[1, ::2] = NINF
    z[2, ::2] = torch.finfo(DT[dtype]).min
    z[3] = torch.finfo(DT[dtype]).min
    z[4, 1:] -= 3000
    t = torch.tensor([vocab, vocab + 7, vocab, vocab, vocab], device="cuda")
    r = logprobs.token_logprobs(z, t)
    assert (r.lse.abs() >= 1024).all()
    a = torch.full((5,), 0.5, device="cuda")
    got = logprobs.token_logprobs_backward(z, t, r.lse, r.entropy, a, a, a)
    assert torch.isnan(got).all()
    got = logprobs.token_logprobs_backward(z, t, r.lse, r.entropy, None, a, a)      # the target plays no part
    check_backward(z, t, r.lse, r.entropy, None, a, a, got)


def test_masked_target():
    """logprob = -inf; its gradient at the target is the upstream one (p = 0 there), the other masked entries get 0."""
    z = torch.randn(2, 300, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    z[:, 100:200] = NINF
    t = torch.tensor([150, 20], device="cuda")
    r = logprobs.token_logprobs(z, t)
    a = torch.tensor([0.25, -0.5], device="cuda")
    g = logprobs.token_logprobs_backward(z, t, r.lse, grad_logprob=a)
    assert float(r.logprob[0]) == NINF and float(g[0, 150]) == 0.25
    g[0, 150] = 0
    assert (g[:, 100:200] == 0).all()
    check_backward(z, t, r.lse, r.entropy, a, None, None, logprobs.token_logprobs_backward(z, t, r.lse, grad_logprob=a))


@pytest.mark.parametrize("shift", [0, 100, 500, 1000, 1015, 1100, 5000, -1000, -5000])
def test_gradient_of_shifted_rows_end_to_end(shift):
    gen = torch.Generator("cuda").manual_seed(abs(shift))
    rows, vocab = 3, 2000
    z = torch.randn(rows, vocab, device="cuda", generator=gen) * 3 + shift
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
    a, b, c = (torch.randn(rows, device="cuda", generator=gen) for _ in range(3))
    r = logprobs.token_logprobs(z, t)
    got = logprobs.token_logprobs_backward(z, t, r.lse, r.entropy, a, b, c).double().cpu()
    zd = z.double().cpu()
    zd0 = zd - shift                                           # exact in float64; the gradient does not depend on the shift
    exact = R.logprobs(zd0, t.cpu())
    av, bv, cv = (v.double().cpu()[:, None] for v in (a, b, c))
    want = R.logprobs_grad(zd0, t.cpu(), exact["lse"], exact["entropy"], av[:, 0], bv[:, 0], cv[:, 0])
    d = torch.log_softmax(zd0, -1)
    h = exact["entropy"][:, None]
    lse = exact["lse"][:, None] + shift
    half_ulp = torch.where(lse.abs() < 1024, torch.exp2(torch.floor(torch.log2(lse.abs())) - 24), torch.zeros_like(lse))
    off = 2e-5 + half_ulp
    bracket = av.abs() + bv.abs() + cv.abs() * (h + d.abs())
    tol = torch.exp(d) * (bracket * (2 ** -21 + d.abs() * 2 ** -22 + off) + cv.abs() * (off + 2e-5 * (1 + h))) + 1e-37
    tol.scatter_add_(1, t.cpu()[:, None], av.abs() * 2 ** -22)
    worst = float(((got - want).abs() / tol).max())
    assert worst <= 1 and not math.isnan(worst), worst
