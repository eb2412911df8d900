"""Host side of the serving calls: refusals that need no device."""
from tests.test_library_host import B  # noqa: F401  (the fixture that loads the library)


def test_planning_in_place_without_a_context_is_refused(B):  # noqa: F811
    assert B.load().dx_pages_plan_in_place(None, 1, 1, 16, 1, 1, *[None] * 10) == B.DX_ERR_INVALID


def test_verification_of_a_planned_step_without_a_context_is_refused(B):  # noqa: F811
    assert B.load().dx_draft_verify_planned(None, None, None, None, None, None, 1, 0, 0, 8, None, None, None, None, None) == B.DX_ERR_INVALID
