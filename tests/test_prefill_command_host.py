"""What the prefill-cost command says of its constant, without a device."""
import json
import types

import numpy as np
import pytest


@pytest.mark.parametrize("more, other, included", [([], 0.0, False), (["--other-us", "0"], 0.0, False), (["--other-us", "2.5"], 2.5e-6, True)])
def test_the_output_says_what_the_constant_holds(monkeypatch, capsys, more, other, included):
    """Attention and the cache's upkeep are measured; the products with the weights are
    the caller's figure, and the output says when there is none."""
    from paper_2603_08739_amd import host
    from paper_2603_08739_amd import prefill_cost as P
    costs = []
    done = dict(requests=24, steps=2, cached_tokens=5, new_tokens=1000, plan_s=1e-3, append_s=2e-3, attention_s=3e-3)
    monkeypatch.setattr(P, "measure", lambda *a, **kw: dict(done))
    monkeypatch.setattr(host, "load", lambda trace: types.SimpleNamespace(free=lambda: None))

    def evaluate(handle, cfgs, cost, groups):
        costs.append(cost["t_prefill_per_token"])
        return None, np.zeros((64, 3))
    monkeypatch.setattr(host, "evaluate", evaluate)
    monkeypatch.setattr(host, "pareto", lambda obj: (np.ones(64, bool), 64))
    P.main(["--requests", "24", "--layers", "2", *more])
    said = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    want = (1e-3 + 2 * 5e-3) / 1000 + other
    assert said["t_prefill_per_token"] == costs[0] == pytest.approx(want, rel=1e-12)
    assert said["layers"] == 2 and said["other_s_per_token"] == pytest.approx(other)
    assert "attention" in said["t_prefill_per_token_holds"]
    assert ("without the products with the weights" in said["t_prefill_per_token_holds"]) == (not included)
