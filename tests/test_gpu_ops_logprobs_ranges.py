"""Gradient of the token log probabilities at the ends of its range: large upstream gradients over masked entries, targets that are
masked, and targets outside the vocabulary in rows of extreme magnitudes.

Masked entries: p = 0, so the gradient is 0 exactly, however large the upstream gradients are; the other entries have the tolerance
of test_gpu_ops_logprobs.check_backward."""
import pytest
import torch

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
