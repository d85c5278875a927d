"""Waits of the paged attention kernels that run out. A limit of a few clocks is kept by polling, so that ordinary waits (for a copy, for another warp) run out at ever
other places: the kernels wind down and report it, and the next call gives what it always gives."""
import pytest
import torch

from paper_2410_05265_b200 import binding

from test_gpu_paged_serving import SCALE, Loop

pytestmark = pytest.mark.gpu
PQ_ERR_TIMEOUT = 6
# lengths, new tokens, heads: single tokens with a worker to a pair (clusters of eight and sixteen, one CTA), in equal stretches of small caches and of one larger than the
# L2, prompts whole and shared by workers, both kernels in one call
CASES = {"one": ([700], [1], 8, 2), "long": ([20000], [1], 8, 2), "pairs": ([300 + i for i in range(200)], [1] * 200, 8, 2), "uneven": ([30000, 40, 9000, 700], [1] * 4, 8, 2),
         "stretches": ([900 + 19 * i for i in range(150)], [1] * 150, 8, 8), "prompt": ([3000], [700], 8, 2),
         "prompts": ([40 + i for i in range(90)], [2 + i % 39 for i in range(90)], 8, 2), "mixed": ([300, 0, 17, 4000], [40, 130, 1, 3], 8, 2)}
SURE = ("stretches", "prompt", "prompts", "mixed")  # the warps of the others find their copies there at the first look


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context()
    yield c
    c.set_wait_limit(0)
    c.check()
    c.close()


@pytest.mark.parametrize("steps", ["head", "vector"])
@pytest.mark.parametrize("name", list(CASES))
def test_waits_that_run_out(ctx, name, steps):
    lengths, new, Hq, Hkv = CASES[name]
    loop = Loop(ctx, steps, lengths, new, Hq, Hkv, spare=sum(new) // 16 + len(new) + 60)
    loop.step()
    ctx.check()
    n = sum(new)
    good = loop.out[:n].clone()

    def attend(limit):
        ctx.set_wait_limit(limit)
        loop.out.fill_(7.0)
        ctx.attn_kv4_paged(loop.cache, loop.q, loop.plan[0], loop.most, SCALE, loop.ws, out=loop.out)
        ctx.set_wait_limit(0)
        status = ctx.check_status()
        assert ctx.check_status() == 0  # reading the status word clears it
        assert (loop.out[n:] == 7.0).all()
        return status

    seen = []
    for limit in (1, 16, 100, 300, 1000, 2000, 5000, 16000):
        for _ in range(4):
            seen.append(attend(limit))
            assert seen[-1] in (0, PQ_ERR_TIMEOUT)
            assert seen[-1] == PQ_ERR_TIMEOUT or torch.equal(loop.out[:n], good)  # what is not reported is right
            assert attend(0) == 0 and torch.equal(loop.out[:n], good)
    assert name not in SURE or PQ_ERR_TIMEOUT in seen[:8], "no limit of a few clocks ran out"
    print(name, steps, "timeouts of four calls by limit:", [sum(s != 0 for s in seen[i: i + 4]) for i in range(0, len(seen), 4)])
