"""examples/generate.py: the steps of a batch behind a prompt give the logits that the whole sequences give as prompts of their own, where nothing is
cut (a threshold of zero keeps every neuron)."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def generate():
    spec = importlib.util.spec_from_file_location("generate", os.path.join(ROOT, "examples", "generate.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("prompt,steps", [(300, 9), (60, 80)])       # longer and shorter than the window, which the steps pass
def test_steps_agree_with_whole_prompts(generate, prompt, steps):
    model = generate.Model(window=64)
    B = 3
    g = torch.Generator().manual_seed(5)
    shared = torch.randint(model.V, (prompt,), generator=g).to(model.dev)
    tails = torch.randint(model.V, (B, steps), generator=g).to(model.dev)
    gen = generate.Generator(model, shared, B, steps, 0.0)
    gen.tau_base.zero_()
    logits = [gen.step(tails[:, i].to(torch.int32)) for i in range(steps)]
    for b in range(B):
        for n in (1, steps):
            whole = generate.Generator(model, torch.cat([shared, tails[b, :n]]), 1, 1, 0.0).logits[0]
            # bf16 hidden states through four layers, rounded in other places on the two ways: a few units of 2^-8 of the logits' size
            rel = (logits[n - 1][b] - whole).norm() / whole.norm()
            assert rel < 8 * 2.0 ** -8, (b, n, float(rel))


def test_a_sparse_run_is_reproducible(generate):
    model = generate.Model()
    prompt = torch.arange(200, device=model.dev) % model.V
    runs = []
    for _ in range(2):
        gen = generate.Generator(model, prompt, 2, 5, 0.45)
        for _ in range(5):
            gen.step(gen.logits.argmax(-1).to(torch.int32))
        runs.append(gen.logits)
    assert torch.equal(runs[0], runs[1]) and torch.isfinite(runs[0]).all()
