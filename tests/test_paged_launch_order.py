"""The paged KV4 kernels under programmatic dependent launch, read from the sources, and the device check of their binding."""
import re

import pytest
import torch

from paper_2410_05265_b200 import binding

from test_launch_order import TRIGGER, kernel_body


@pytest.mark.parametrize("name", ["page_plan_kernel", "page_release_kernel"])
def test_writers_of_tables_and_lengths_never_trigger(name):
    """Another kernel may read lengths and tables ahead of its own wait."""
    assert not TRIGGER.search(kernel_body("pq_pages.cu", name))


def test_the_append_never_triggers():
    body = kernel_body("pq_qk_rope.cu", "qk_norm_rope_kernel")
    assert [m.group(0) for m in re.finditer(r"[^\n;{}]*(?:launch_dependents|pdl_trigger)", body)] == ["  if (!APPEND) pq::pdl_trigger"]


@pytest.mark.parametrize("source,name", [
    ("pq_pages.cu", "page_plan_kernel"), ("pq_pages.cu", "page_release_kernel"), ("pq_qk_rope.cu", "qk_norm_rope_kernel"),
    ("pq_qk_rope.cu", "kv4_paged_read_kernel"), ("pq_paged_decode.cu", "paged_decode_kernel"),
])
def test_the_wait_comes_before_every_read_and_before_the_trigger(source, name):
    body = kernel_body(source, name)
    wait = body.index("pdl_wait")
    first = re.search(r"ld_dep|__ldcg|\bbulk_load|atomicAdd|report\(", body)
    assert first is None or wait < first.start()
    trigger = TRIGGER.search(body)
    assert trigger is None or wait < trigger.start()
    assert "__ldg(" not in body and "ld.global.nc" not in body


def test_the_kernel_for_several_rows_waits_last_and_never_triggers():
    """It starts behind the wait of the kernel for single tokens, which always precedes it, and must not end before that one."""
    body = kernel_body("pq_paged_prefill.cu", "paged_prefill_kernel")
    assert not TRIGGER.search(body) and body.count("pdl_wait") == 1
    assert re.search(r"pq::pdl_wait\(\);\s*}$", body) and "__ldg(" not in body and "ld.global.nc" not in body
    # in the wait's place a fence ahead of the first read
    assert body.index("__threadfence()") < body.index("ld_dep(")
    # no thread returns ahead of it: what returns are lambdas
    assert len(re.findall(r"^  (?:if \(.*\) )?return;", body, re.M)) == 0


class _Elsewhere:
    device = torch.device("cuda:1")

    def get_device(self):
        return 1


def test_tensors_of_another_device_and_another_current_device_are_refused(monkeypatch):
    ctx = binding.Context.__new__(binding.Context)
    ctx.device = 0
    current = [0]
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    here = type("Here", (_Elsewhere,), {"get_device": lambda self: 0})()
    ctx._here(here, None)
    with pytest.raises(ValueError):
        ctx._here(here, _Elsewhere())
    with pytest.raises(ValueError):
        ctx._here(torch.zeros(1))
    current[0] = 1
    with pytest.raises(ValueError):
        ctx._here(here)
