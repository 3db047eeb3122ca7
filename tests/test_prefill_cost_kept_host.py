"""The measured prefill cost over a quantised cache, without a device: what it makes and
what it refuses."""
import types

import pytest
import torch

import tracegen as tg
from tests.test_prefill_memory_host import Event


@pytest.mark.parametrize("kept, held", [("16", torch.bfloat16), ("fp8", torch.float8_e4m3fn), ("i8", torch.int8)])
def test_the_cache_holds_what_is_asked_for(monkeypatch, kept, held):
    from paper_2603_08739_amd import prefill_cost as P
    made = []
    plan = lambda *a, **kw: types.SimpleNamespace(result=torch.zeros(4, dtype=torch.int32))  # noqa: E731
    monkeypatch.setattr(P, "kvpaged", types.SimpleNamespace(
        Plan=plan, Cache=lambda *a, **kw: made.append((a, kw)), Rope=lambda dim, base: types.SimpleNamespace(free=lambda: None),
        KV_PAGED_MAX_TOKENS=524288, kv_paged_plan=lambda *a: None, kv_paged_append=lambda *a, **kw: None, kv_paged_attention=lambda *a, **kw: None))
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    P.measure(tg.tiny(n_req=4), 400, batch=4, q_heads=2, kv_heads=1, head_dim=16, device="cpu", kept=kept)
    (tensors, more), = made
    assert tensors[0].dtype == tensors[1].dtype == held and tensors[0].shape == (400, 1, 16, 16)
    if kept == "16":
        assert len(tensors) == 2 and not more
    else:
        assert more == dict(block_scales=True) and all(s.shape == (400, 1) and s.dtype == torch.float32 for s in tensors[2:])


@pytest.mark.parametrize("kept", ["8", "int8", None, ""])
def test_other_caches_are_refused(kept):
    from paper_2603_08739_amd import prefill_cost as P
    with pytest.raises(ValueError, match="kept"):
        P.measure(tg.tiny(n_req=4), 400, kept=kept, device="cpu")


def test_the_command_refuses_other_caches(capsys):
    from paper_2603_08739_amd import prefill_cost as P
    with pytest.raises(SystemExit):
        P.main(["--cache", "4"])
    assert "--cache" in capsys.readouterr().err
