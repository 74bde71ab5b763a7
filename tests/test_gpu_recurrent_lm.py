"""The example model trains, and says the same token by token as all at once."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    spec = importlib.util.spec_from_file_location("recurrent_lm", os.path.join(ROOT, "examples", "recurrent_lm.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_it_learns(example, dtype):
    model = example.RecurrentLM(32, 64, 2, dtype=dtype)
    losses = example.train(model, 60, vocab=32, rows=8, length=150)
    assert all(v == v for v in losses)
    # from a uniform guess, log 32 = 3.47
    assert sum(losses[-5:]) / 5 < 0.7 * sum(losses[:3]) / 3


def test_steps_say_what_the_prompt_says(example):
    model = example.RecurrentLM(50, 96, 3)
    ids = torch.randint(0, 50, (5, 23), device="cuda")
    with torch.no_grad():
        whole = model.forward(ids)
        states = []
        model.forward(ids[:, :9], states=states)
        for k in range(9, 23):
            logits = model.step(ids[:, k], states)
            assert torch.allclose(logits, whole[:, k], rtol=1e-3, atol=1e-3 * float(whole.std())), k


def test_packed_documents_do_not_see_each_other(example):
    model = example.RecurrentLM(50, 64, 2)
    ids = torch.randint(0, 50, (1, 80), device="cuda")
    starts = torch.zeros(1, 80, dtype=torch.bool, device="cuda")
    starts[0, 33] = True
    with torch.no_grad():
        packed = model.forward(ids, starts)
        alone = model.forward(ids[:, 33:].contiguous())
    assert torch.allclose(packed[:, 33:], alone, rtol=1e-3, atol=1e-3 * float(alone.std()))
