"""What the serving loop's pools are to a program that looks into them, without a GPU."""
import types

import pytest
import torch

import paper_2410_18248_amd as P
from paper_2410_18248_amd import engine


@pytest.mark.parametrize("dtype,held", [(P.LAMPS_F32, torch.float32), (P.LAMPS_BF16, torch.bfloat16), (P.LAMPS_E4M3, torch.uint8)])
def test_pools_have_the_type_of_what_they_hold(monkeypatch, dtype, held):
    """Elements of the rows' own type, [block][layer][kv head][tile]; codes and scales are bytes."""
    stub = types.SimpleNamespace(cuda_stream=0, destroy=lambda: None)
    monkeypatch.setattr(torch.cuda, "Stream", lambda device: stub)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    monkeypatch.setattr(engine.P, "Lamps", lambda cfg, *args: stub)
    monkeypatch.setattr(engine.P, "LampsSched", lambda cfg: stub)
    cfg = P.LampsConfig(2, 4, 2, 64, 16, 8, 4, 4, dtype)
    eng = engine.LiveEngine(cfg, types.SimpleNamespace(memory_tokens=128, max_batch=4), None, "cpu")
    for pool in (eng.k_pool, eng.v_pool):
        assert pool.dtype == held and pool.numel() * pool.element_size() == P.lamps_pool_bytes(cfg)
    if held != torch.uint8:
        assert eng.k_pool.view(8, 2, 2, 16 * 64).dtype == eng.tdtype == held
