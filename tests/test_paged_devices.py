"""A block table or a cache on another device than the context's is refused by every paged call, before the library is called. Needs no GPU: the objects only say
where they are."""
import pytest
import torch

from paper_2410_05265_b200 import binding


class Fake:
    """A CUDA tensor of that type and shape that says it is on cuda:`at`."""
    is_cuda = True

    def __init__(self, dtype, shape, at):
        self.dtype, self.shape, self.at, self.device = dtype, torch.Size(shape), at, torch.device("cuda", at)

    def get_device(self):
        return self.at

    def is_contiguous(self):
        return True

    def stride(self):
        return tuple(torch.empty(self.shape, device="meta").stride())

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 1 << 20


def pages_on(at):
    i32 = lambda *shape: Fake(torch.int32, shape, at)
    return binding.Pages(i32(2, 4), i32(2), i32(10), i32(1), 16)


def cache_on(at):
    return binding.KV4PagedCache(pages_on(at), None, None, Fake(torch.uint8, (10, 2, 2, 16, 64), at), 4, s_k=Fake(torch.float32, (2,), at),
                                 s_v=Fake(torch.float32, (2,), at))


@pytest.fixture
def ctx(monkeypatch):
    c = binding.Context.__new__(binding.Context)
    called = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: called.append(name) or 0

    c.lib, c.h, c.device, c.called = Library(), None, 0, called
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    yield c
    c.h = None


def calls(ctx, at):
    """Every paged call, its own tensors on cuda:0, the table or the cache on cuda:`at`."""
    t = lambda dtype, *shape: Fake(dtype, shape, 0)
    i32, i64, bf16, u8 = torch.int32, torch.int64, torch.bfloat16, torch.uint8
    return {
        "pq_page_plan": lambda: ctx.page_plan(pages_on(at), t(i32, 2), out=(t(i32, 3), t(i64, 5), t(i32, 5))),
        "pq_page_release": lambda: ctx.page_release(pages_on(at), t(i32, 2)),
        "pq_qk_norm_rope_kv4_paged_append": lambda: ctx.qk_norm_rope_kv4_paged_append(cache_on(at), t(bf16, 5, 8 * 128), None, None, 0.0, t(i32, 5), t(i64, 5), 1e4,
                                                                                      q_out=t(bf16, 5, 4, 128)),
        "pq_kv4_paged_read": lambda: ctx.kv4_paged_read(cache_on(at), t(i64, 5), out=t(bf16, 5, 2, 2, 128)),
        "pq_attn_kv4_paged": lambda: ctx.attn_kv4_paged(cache_on(at), t(bf16, 5, 4, 128), t(i32, 3), 3, 0.1, t(u8, 100), out=t(bf16, 5, 4, 128)),
    }


@pytest.mark.parametrize("name", ["pq_page_plan", "pq_page_release", "pq_qk_norm_rope_kv4_paged_append", "pq_kv4_paged_read", "pq_attn_kv4_paged"])
def test_a_cache_of_another_device_is_refused(ctx, name):
    calls(ctx, 0)[name]()
    assert ctx.called == [name]  # in order: the library is called
    with pytest.raises(ValueError):
        calls(ctx, 1)[name]()
    assert ctx.called == [name]


def test_a_cache_in_two_places_is_refused():
    pg = pages_on(0)
    with pytest.raises(AssertionError):
        binding.KV4PagedCache(pg, None, None, Fake(torch.uint8, (10, 2, 2, 16, 64), 1), 4, s_k=Fake(torch.float32, (2,), 0), s_v=Fake(torch.float32, (2,), 0))
