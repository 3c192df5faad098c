"""Host check of the 8-bit LM head's launch plans, compiled for the host from the library's own headers."""

from test_host_checks import _run_host_check


def test_every_launch_form_is_made_and_covers_the_ids(tmp_path):
    _run_host_check(tmp_path, "q8_plan_check")
