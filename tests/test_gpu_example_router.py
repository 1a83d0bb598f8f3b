"""The router fine-tuning example runs the new calls together and does what it says."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "router_finetune_mx4.py")


def test_router_finetune_balances_the_load():
    print("CASE example", flush=True)
    spec = importlib.util.spec_from_file_location("router_finetune_mx4", PATH)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    first, last = ex.train(steps=30, T=512, H=512, I=256, E=16, k=2)
    assert first["task"] == 0.0 and first["load"] > 2.0
    assert last["balance"] < 0.8 * first["balance"] and last["load"] < 0.8 * first["load"]
