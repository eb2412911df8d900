"""Host side of the serving calls: refusals that need no device."""
import pytest
import torch

from tests.test_library_host import B  # noqa: F401  (the fixture that loads the library)


def test_planning_in_place_without_a_context_is_refused(B):  # noqa: F811
    assert B.load().dx_pages_plan_in_place(None, 1, 1, 16, 1, 1, *[None] * 10) == B.DX_ERR_INVALID


def test_verification_of_a_planned_step_without_a_context_is_refused(B):  # noqa: F811
    assert B.load().dx_draft_verify_planned(None, None, None, None, None, None, 1, 0, 0, 8, None, None, None, None, None) == B.DX_ERR_INVALID


def test_tensors_in_host_memory_are_refused(B):  # noqa: F811
    """The kernels read the addresses as they are: a tensor on the CPU must not get that far."""
    class Library:
        def __getattr__(self, name):
            return lambda *args: pytest.fail(f"{name} was called")

    ctx = object.__new__(B.Context)
    ctx.lib, ctx.h = Library(), None
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    rows, p = torch.zeros((3, 2, 64), dtype=torch.bfloat16), torch.zeros((5, 8))
    cache = B.DxKvCache(16, 16, None, None, 2, 64, 16, 4, 0, 0)
    drafts = (p, None, ints(3), ints(3), 3, p[0, :3].contiguous(), p[0, :2].contiguous(), ints(2, 4), ints(2), ints(2))
    calls = [lambda: ctx.dx_pages_plan(ints(2), ints(2), None, ints(1), ints(4), ints(2, 3), 16, ints(2), ints(1), ints(3), ints(3), ints(3), ints(4)),
             lambda: ctx.dx_pages_plan_in_place(ints(2), ints(2), ints(2), ints(1), ints(4), ints(2, 3), 16, ints(3), ints(3), ints(3), ints(4)),
             lambda: ctx.dx_kv_write(cache, rows, rows, ints(3)),
             lambda: ctx.dx_paged_attention(cache, rows, ints(3), ints(2), ints(2, 3), 2, 0.1, 0, rows),
             lambda: ctx.dx_draft_verify(*drafts), lambda: ctx.dx_draft_verify_planned(ints(4), *drafts)]
    for call in calls:
        with pytest.raises(AssertionError, match="on the device"):
            call()
    k = torch.zeros((4, 2, 8, 16, 8), dtype=torch.bfloat16)
    with pytest.raises(AssertionError, match="on the device"):
        B.make_kv_cache(k, torch.zeros((4, 2, 2, 64, 8), dtype=torch.bfloat16))
