"""Refusals of the expert layer's self-test (runs without a GPU; nothing is enqueued by it)."""
import pytest

import paper_2208_10391_b200 as mom


@pytest.mark.parametrize("limit_ms", [0.0, -5.0, 1000.5, float("nan"), float("inf")])
def test_moe_probe_limits(limit_ms):
    plan = mom.mom_moe_plan(64, 32, 8, 2, mom.BF16, mom.BF16)
    with pytest.raises(mom.MomError) as e:
        plan.probe_wait_timeout(limit_ms)
    assert e.value.status == mom.ERR_INVALID_ARG


def test_moe_probe_accepts_and_enqueues_nothing():
    plan = mom.mom_moe_plan(64, 32, 8, 2, mom.BF16, mom.BF16)
    plan.probe_wait_timeout(1000.0)
    assert plan.device_status() == (0, 0)
    assert mom._lib.mom_moe_probe_wait_timeout(None, 1.0) == mom.ERR_INVALID_ARG
