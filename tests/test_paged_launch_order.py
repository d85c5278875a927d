"""The paged KV4 kernels under programmatic dependent launch, read from the sources, and the device check of their binding."""
import os
import re

import pytest
import torch

from paper_2410_05265_b200 import binding

from test_launch_order import CSRC, TRIGGER, kernel_body


def source(name):
    return os.path.join(CSRC, name)


@pytest.mark.parametrize("name", ["page_plan_kernel", "page_release_kernel"])
def test_writers_of_tables_and_lengths_never_trigger(name):
    """Another kernel may read lengths and tables ahead of its own wait."""
    assert not TRIGGER.search(kernel_body("pq_pages.cu", name))


def test_the_append_never_triggers():
    body = kernel_body("pq_qk_rope.cu", "qk_norm_rope_kernel")
    assert [m.group(0) for m in re.finditer(r"[^\n;{}]*(?:launch_dependents|pdl_trigger)", body)] == ["  if (!APPEND) pq::pdl_trigger"]


@pytest.mark.parametrize("source,name", [
    ("pq_pages.cu", "page_plan_kernel"), ("pq_pages.cu", "page_release_kernel"), ("pq_qk_rope.cu", "qk_norm_rope_kernel"),
    ("pq_qk_rope.cu", "kv4_paged_read_kernel"), ("pq_paged_prefill.cu", "paged_prefill_kernel"),
])
def test_the_wait_comes_before_every_read_and_before_the_trigger(source, name):
    body = kernel_body(source, name)
    wait = body.index("pdl_wait")
    first = re.search(r"ld_dep|__ldcg|\bbulk_load|atomicAdd|report\(", body)
    assert first is None or wait < first.start()
    trigger = TRIGGER.search(body)
    assert trigger is None or wait < trigger.start()
    assert "__ldg(" not in body and "ld.global.nc" not in body


def test_the_kernel_for_single_tokens_ends_behind_the_one_for_several_rows():
    """Alone it waits before it reads anything. Behind the kernel for several rows, which always precedes it then, it reads without a wait of its own (a fence
    in its place), never triggers, and its last CTA waits on every way out."""
    body = kernel_body("pq_paged_decode.cu", "paged_decode_kernel")
    start = re.search(r"if \(beside\) \{\s*__threadfence\(\);\s*\} else \{\s*pq::pdl_wait\(\);\s*pq::pdl_trigger\(\);\s*\}", body)
    assert start and "const bool beside = p.max_new > 1;" in body[: start.start()]
    first = re.search(r"ld_dep|__ldcg|\bbulk_load|atomicAdd|report\(", body)
    assert start.end() < first.start() and "__ldg(" not in body and "ld.global.nc" not in body
    assert len(TRIGGER.findall(body)) == 1
    assert re.search(r"auto leave = \[&\]\(\) \{\s*if \(beside && blockIdx.x == gridDim.x - 1\) pq::pdl_wait\(\);\s*\};", body)
    assert re.search(r"leave\(\);\s*}$", body)
    assert body.count("return leave();") == 3 and re.findall(r"^ {2,4}(?:if \(.*\) )?return;", body, re.M) == ["    if (!is_ok) return;"]  # (a lambda's)
    with open(source("pq_paged_attn.cu")) as f:
        text = f.read()
    assert text.index("pq_paged_prefill_launch(") < text.index("return pq_paged_decode_launch(")


def test_tensors_of_another_device_and_another_current_device_are_refused(monkeypatch):
    ctx = binding.Context.__new__(binding.Context)
    ctx.device = 0
    current = [0]
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    assert ctx._here() == 0

    class Fake:
        """An int32 vector that says it is on cuda:`at`."""
        dtype, is_cuda, shape, device = torch.int32, True, torch.Size([4]), "cuda"
        at = 0
        get_device = lambda self: self.at
        is_contiguous = lambda self: True
        stride = lambda self: (1,)
        data_ptr = lambda self: 64

    here, there = Fake(), Fake()
    there.at = 1
    assert binding._arr(here, torch.int32, (4,), 0, "t") == 64
    with pytest.raises(ValueError):
        binding._arr(there, torch.int32, (4,), 0, "t")
    with pytest.raises(TypeError):
        binding._arr(torch.zeros(4, dtype=torch.int32), torch.int32, (4,), 0, "t")
    with pytest.raises(TypeError):
        binding._arr(here, torch.int64, (4,), 0, "t")
    with pytest.raises(AssertionError):
        binding._arr(here, torch.int32, (5,), 0, "t")
    current[0] = 1
    with pytest.raises(ValueError):
        ctx._here()
