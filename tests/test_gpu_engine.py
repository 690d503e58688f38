"""The engine's iterations on the paged cache: pages in use are the projected
KV blocks, and its attention is the same as over one unpaged sequence."""
import numpy as np
import pytest
import torch

import oracle
from paper_2408_05235_amd import configs, synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block_tokens", [16, 24])
def test_pages_in_use_are_the_projected_blocks(gpu, block_tokens):
    from paper_2408_05235_amd.engine import Engine
    inp = synth.make_inputs(synth.scaled(configs.get_config(0), n_scenarios=1))
    inp["block_tokens"] = block_tokens
    proj = oracle.project(inp)
    e = Engine(inp["prompt"], inp["generated"], inp["remaining"], block_tokens, int(inp["kv_capacity"][0]))
    e.prefill()
    used = [e.cache.pages_used()]
    for _ in range(120):
        x = e.step()
        used.append(e.cache.pages_used())
    assert bool(torch.isfinite(x).all())
    assert np.array_equal(torch.stack(used).cpu().numpy(), proj["kv"][0, :121])


def test_command(gpu, capsys):
    from paper_2408_05235_amd import engine
    engine.main(["--iterations", "40", "--layers", "2", "--window", "256", "--sinks", "4"])
    assert "iterations/s" in capsys.readouterr().out
