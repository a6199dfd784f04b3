"""Gradient of the token log probabilities at the ends of its range.

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
