"""The operators' calls keep nothing between them: several streams at once, and several host threads, give the bits of one after
the other."""
import threading

import pytest
import torch

from paper_2502_11034_b200 import act8, logprobs

pytestmark = pytest.mark.gpu


def work(seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dy = (torch.randn(2500, 1100, device="cuda", generator=gen) * 1e-2).bfloat16()
    x = torch.randn(2500, 900, device="cuda", generator=gen).bfloat16()
    z = (torch.randn(70, 30001, device="cuda", generator=gen) * 3).bfloat16()
    t = torch.randint(0, 30001, (70,), device="cuda", generator=gen)
    a = torch.full((70,), 0.1, device="cuda")

    def calls(stream=None):
        x8 = act8.encode(x, stream=stream)
        r = logprobs.token_logprobs(z, t, top_k=9, stream=stream)
        big = act8.linear_wgrad(dy, x8, stream=stream)
        h, g8, u8 = act8.swiglu(x[:, :450], x[:, 450:], stream=stream)
        low = act8.linear_wgrad(dy, x8, torch.bfloat16, stream=stream)
        act8.linear_wgrad(dy, x8, out=big, accumulate=True, stream=stream)
        g = logprobs.token_logprobs_backward(z, t, r.lse, r.entropy, a, a, a, stream=stream)
        return [big, low, h, act8.decode(g8, stream=stream), g, *r]

    return calls


def test_streams_that_overlap():
    jobs = [work(i) for i in range(3)]
    alone = []
    for job in jobs:
        alone.append(job())
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        got = [job(s) for job, s in zip(jobs, streams)]
        torch.cuda.synchronize()
        for x, y in zip(got, alone):
            assert all(torch.equal(p, q) for p, q in zip(x, y))


def test_threads_that_call_at_once():
    jobs = [work(10 + i) for i in range(4)]
    alone = [job() for job in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got, errors = [None] * len(jobs), []
    start = threading.Barrier(len(jobs))

    def one(i):
        try:
            start.wait(30)
            for _ in range(4):
                got[i] = jobs[i](streams[i])
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=one, args=(i,)) for i in range(len(jobs))]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for x, y in zip(got, alone):
        assert all(torch.equal(p, q) for p, q in zip(x, y))
