"""What the measured prefill cost keeps while it runs, without a device: the operators
are played by stand-ins that count the plans alive."""
import gc
import types
import weakref

import pytest
import torch

import tracegen as tg


class Event:
    def __init__(self, enable_timing=False):
        pass

    def record(self):
        pass

    def elapsed_time(self, other):
        return 1.0


@pytest.fixture
def operators(monkeypatch):
    from paper_2603_08739_amd import prefill_cost as P
    plans, most = [], [0]

    class Plan:
        def __init__(self, *a, **kw):
            gc.collect()
            most[0] = max(most[0], sum(p() is not None for p in plans))
            plans.append(weakref.ref(self))
            self.work = bytearray(100)
            self.result = torch.zeros(4, dtype=torch.int32)

    fake = types.SimpleNamespace(
        Plan=Plan, Cache=lambda k, v: None, Rope=lambda dim, base: types.SimpleNamespace(free=lambda: None), KV_PAGED_MAX_TOKENS=524288,
        kv_paged_plan=lambda *a: None, kv_paged_append=lambda *a, **kw: None, kv_paged_attention=lambda *a, **kw: None)
    monkeypatch.setattr(P, "kvpaged", fake)
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    return P, plans, most


def test_plans_are_not_kept_until_the_end(operators):
    """A plan's work memory is tens of megabytes; a trace has thousands of steps."""
    P, plans, most = operators
    done = P.measure(tg.tiny(n_req=60), 4000, batch=4, q_heads=2, kv_heads=1, head_dim=16, device="cpu")
    assert done["steps"] == len(plans) == 15 and most[0] <= 1
    assert done["plan_s"] == done["append_s"] == pytest.approx(0.015)


def test_a_refused_plan_of_any_step_is_reported(operators, monkeypatch):
    P, plans, most = operators

    def flagged(plan, *a):
        plan.result[3] = 1 if len(plans) == 2 else 0
    monkeypatch.setattr(P.kvpaged, "kv_paged_plan", flagged)
    with pytest.raises(RuntimeError, match="refused"):
        P.measure(tg.tiny(n_req=60), 4000, batch=4, q_heads=2, kv_heads=1, head_dim=16, device="cpu")
