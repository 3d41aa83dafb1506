"""The operators of a training step together, as the examples use them."""
import importlib.util
import os

import pytest
import torch

from paper_2509_04084_amd import lowdiff as ld

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example(name):
    spec = importlib.util.spec_from_file_location(name, os.path.join(ROOT, "examples", name + ".py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("steps,window", [(1, 1), (9, 4), (12, 12), (7, 1)])
def test_a_model_of_both_optimizers_is_recovered(steps, window):
    losses, same = example("muon_recovery").train(steps=steps, window=window)
    assert len(losses) == steps and all(x == x and x < 100 for x in losses) and same


def test_the_examples_gradients():
    """Against autograd's of the same loss in 64 bits. Sums of up to 256 terms, products of three such in a row: 3 * 256 roundings of 2^-24 of
    the sum of magnitudes are 5e-5 of it, which is no more than a few times the gradient's own norm."""
    m, g = example("muon_recovery"), torch.Generator().manual_seed(1)
    weights = [torch.randn(*s, generator=g) * 0.3 for s in ((53, 24), (40, 24), (24, 40))]
    tokens = torch.randint(0, 53, (64,), generator=g)
    wanted = torch.randint(0, 53, (64,), generator=g)
    loss, grads = m.gradients([w.to(DEV) for w in weights], tokens.to(DEV), wanted.to(DEV))
    exact = [w.double().requires_grad_() for w in weights]
    table, up, down = exact
    x = table[tokens]
    y = x + torch.relu(x @ up.t()) @ down.t()
    want = torch.nn.functional.cross_entropy(y @ table.t(), wanted)
    want.backward()
    assert abs(loss - float(want.detach())) <= 1e-5 * float(want.detach())
    for a, b in zip(grads, exact):
        assert float((a.double().cpu() - b.grad).norm()) <= 2e-4 * float(b.grad.norm())


def test_a_step_in_a_graph():
    """Log probabilities, gradient and update captured as one, replayed over changing inputs with eager work between."""
    g = torch.Generator(device=DEV).manual_seed(2)
    T, V, d = 96, 1000, 64
    w, m = torch.randn(V, d, generator=g, device=DEV) * 0.1, torch.zeros(V, d, device=DEV)
    x, ids = torch.randn(T, d, generator=g, device=DEV), torch.randint(0, V, (T,), generator=g, device=DEV)
    weight = torch.full((T,), -1.0 / T, device=DEV)

    def step(logits, w, m):
        r = ld.ld_token_logprob(logits, ids, entropy=True, top=3)
        dz = ld.ld_token_logprob_grad(logits, r.stats, ids, weight, r.entropy, weight)
        ld.ld_merge_dense_muon([w], [m], [[dz[:, :d].contiguous()[:64]]], 0.05)
        return [*r, dz]
    state = torch.randn(64, d, generator=g, device=DEV), torch.zeros(64, d, device=DEV)
    logits = x @ w.t()
    step(logits, *[t.clone() for t in state])
    held_state = [t.clone() for t in state]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(logits, *held_state)
    eager = [t.clone() for t in state]
    for a, b in zip(held_state, state):
        a.copy_(b)
    for _ in range(3):
        logits.copy_(torch.randn(T, V, generator=g, device=DEV))
        want = step(logits, *eager)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held + held_state, want + eager):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
