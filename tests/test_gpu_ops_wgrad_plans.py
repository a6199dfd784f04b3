"""The weight gradient's plans and its accuracy.

On B200 a product has 74 pairs of SMs.  240 tiles of 256 x 256 are 222 taken whole, three to a pair (the accumulators' buffers are
used again), and 18 whose tokens are shared out; over 8192 tokens a share is longer than an fp32 result stays in the accumulator, so
partial sums are added onto as well.  74 and 148 tiles are taken whole, fewer are shared out.

Accuracy.  The tensor core cuts when it adds 16 tokens to an accumulator: at most 2^-23 of the running sum each time.  One chain of
1024 / 2048 tokens of normal values was measured at 2e-7 / 4.4e-7 of the result's norm, so chains of 1536 give 3.2e-7; up to 11
rounded additions of them add 2^-25 sqrt(11) = 1e-7.  Where tokens and features have scales of their own the largest tokens decide
and the error may double: 1e-6 of the norm is what the header promises for such values."""
import pytest
import torch

from paper_2502_11034_b200 import act8, binding
from test_gpu_ops_act8 import DT, check_wgrad, wgrad_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,n,k", [(300, 7680, 2048), (8192, 7680, 2048), (8190, 7501, 1900)])
def test_whole_and_shared_out_tiles_in_one_call(tokens, n, k, dtype, accumulate):
    dy, x8 = wgrad_case(tokens, n, k, 13)
    shared = binding.lib().adagc_act8_linear_wgrad_workspace_bytes(tokens, n, k, None, 7680)
    assert shared >= (4 * 18 * 256 * 256 * 4 if tokens > 8000 else 0)
    old = (torch.randn(n, k, device="cuda", generator=torch.Generator("cuda").manual_seed(1)) * 5).to(DT[dtype]) if accumulate else None
    out = None if old is None else old.clone()
    got = act8.linear_wgrad(dy, x8, DT[dtype], out=out, accumulate=accumulate)
    check_wgrad(dy, x8, got, old)
    again = act8.linear_wgrad(dy, x8, DT[dtype], out=None if old is None else old.clone(), accumulate=accumulate)
    assert torch.equal(got, again)


def test_no_tokens_leave_an_accumulated_output_alone():
    dy, x8 = wgrad_case(10, 70, 50, 11)
    for dtype in DT.values():
        out = torch.randn(70, 50, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).to(dtype)
        before = out.clone()
        act8.linear_wgrad(dy[:0], x8[:0], out=out, accumulate=True)
        assert torch.equal(out, before)


@pytest.mark.parametrize("scales", ["equal", "differing"])
@pytest.mark.parametrize("n,k", [(9472, 512), (512, 512)])     # tiles taken whole; tokens shared out
@pytest.mark.parametrize("tokens", [4096, 8192, 16384])
def test_fp32_results_are_within_1e6_of_the_norm(tokens, n, k, scales):
    gen = torch.Generator("cuda").manual_seed(tokens + n)
    dy = (torch.randn(tokens, n, device="cuda", generator=gen) * 1e-3).bfloat16()
    x = torch.randn(tokens, k, device="cuda", generator=gen)
    if scales == "differing":
        x *= (torch.randn(k, device="cuda", generator=gen).abs() + 0.2) * (torch.rand(tokens, 1, device="cuda", generator=gen) + 0.5)
    x8 = act8.encode(x.bfloat16())
    got = act8.linear_wgrad(dy, x8)
    want = dy[:, :256].double().T @ act8.decode(x8, torch.float32).double()
    assert float((got[:256].double() - want).norm() / want.norm()) < 1e-6


@pytest.mark.parametrize("n,k", [(9472, 512), (512, 512)])
def test_fp32_accumulation_rounds_once_onto_what_is_there(n, k):
    """Old values far above the gradient: the sum is off by the one rounding onto them, half an ulp, and the gradient's own error."""
    tokens = 8192
    gen = torch.Generator("cuda").manual_seed(5)
    dy = (torch.randn(tokens, n, device="cuda", generator=gen) * 1e-2).bfloat16()
    x8 = act8.encode(torch.randn(tokens, k, device="cuda", generator=gen).bfloat16())
    alone = act8.linear_wgrad(dy, x8)
    old = torch.rand(n, k, device="cuda", generator=gen) * 2 ** 19 + 2 ** 20        # an ulp is 2^-3 up to 2^21
    out = old.clone()
    act8.linear_wgrad(dy, x8, out=out, accumulate=True)
    off = (out.double() - (old.double() + alone.double())).abs().max()
    assert float(off) <= 2 ** -4 + 2 ** -20 * float(alone.abs().max())


@pytest.mark.parametrize("accumulate", [False, True])
def test_bfloat16_result_over_many_tokens(accumulate):
    """All products positive, the worst case for cutting: a chain of 16384 tokens loses at most 1024 * 2^-23 of the sum, the rounded
    additions of 8 such chains (and of the old value) 9 * 2^-24; then one rounding to bfloat16, half an ulp.  Output features have scales
    of their own, so that the results lie anywhere between two bfloat16 numbers."""
    tokens, n, k = 1 << 17, 9224, 257                                               # 74 tiles, all whole
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    gen = torch.Generator("cuda").manual_seed(6)
    scale = torch.rand(n, device="cuda", generator=gen) / 2 + 0.5
    dy = torch.empty(tokens, n, dtype=torch.bfloat16, device="cuda")
    for part in dy.split(1 << 15):
        part.copy_((torch.rand(part.shape, device="cuda", generator=gen) + 0.5) * scale)
    x8 = act8.encode((torch.rand(tokens, k, device="cuda", generator=gen) + 0.5).bfloat16())
    old = (torch.rand(n, k, device="cuda", generator=gen) * 1e5).bfloat16() if accumulate else None
    got = act8.linear_wgrad(dy, x8, torch.bfloat16, out=None if old is None else old.clone(), accumulate=accumulate)[:256].double()
    want = dy[:, :256].double().T @ act8.decode(x8, torch.float32).double() + (0 if old is None else old[:256].double())
    tol = torch.exp2(torch.floor(torch.log2(want)) - 8) + want * (1024 * 2 ** -23 + 9 * 2 ** -24)
    assert float(((got - want).abs() / tol).max()) <= 1
