"""The loss, the layers and the optimiser together: the class of the optimiser, and the example's training run."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def pkg():
    from paper_2204_00595_amd import autograd, binding, optim
    return autograd, binding, optim


def parameters(dtype=torch.bfloat16, seed=0):
    gen = torch.Generator().manual_seed(seed)
    shapes = [(4, 48, 40), (4, 48, 40), (2, 130, 64), (70, 90), (4, 40, 48)]
    ps = [torch.nn.Parameter((torch.randn(s, generator=gen) / 7).to(dtype).cuda()) for s in shapes]
    for p in ps:
        p.grad = (torch.randn(p.shape, generator=gen) * 1e-2).to(dtype).cuda()
    return ps


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_class_makes_the_steps_of_the_call(pkg, dtype):
    _, binding, optim = pkg
    ps, qs = parameters(dtype), parameters(dtype)
    o = optim.Muon(ps, lr=0.03, momentum=0.9, weight_decay=0.1)
    masters = [q.detach().float() for q in qs]
    momenta = [torch.zeros_like(m) for m in masters]
    for _ in range(3):
        o.step()
        for q, k, v in zip(qs, masters, momenta):
            binding.monarch_muon_step([q.detach()], [q.grad], [v], lr=0.03, momentum=0.9, weight_decay=0.1,
                                      masters=[k] if dtype == torch.bfloat16 else None)
    for p, q, v in zip(ps, qs, momenta):
        assert torch.equal(p, q) and torch.equal(o.state[p]["momentum"], v)
    if dtype == torch.bfloat16:
        assert all(torch.equal(o.state[p]["master"], k) for p, k in zip(ps, masters))


def test_its_state_comes_back_whole(pkg):
    _, _, optim = pkg
    ps = parameters()
    o = optim.Muon(ps, lr=0.03)
    o.step()
    saved = o.state_dict()
    qs = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    n = optim.Muon(qs, lr=0.5)
    n.load_state_dict(saved)
    for p, q in zip(ps, qs):
        q.grad = p.grad.clone()
        assert n.state[q]["momentum"].dtype == torch.float32 and torch.equal(n.state[q]["master"], o.state[p]["master"])
        assert n.state[q]["master"].data_ptr() != o.state[p]["master"].data_ptr()
    o.step()
    n.step()
    assert all(torch.equal(p, q) for p, q in zip(ps, qs))


def test_small_updates_add_up_on_masters(pkg):
    """Updates below half a rounding of a bf16 weight: lost on the weights themselves, kept on fp32 masters."""
    _, _, optim = pkg
    for masters in (True, False):
        p = torch.nn.Parameter(torch.ones((2, 16, 16), dtype=torch.bfloat16, device="cuda"))
        o = optim.Muon([p], lr=1e-3, masters=masters)
        for _ in range(40):
            p.grad = torch.eye(16, dtype=torch.bfloat16, device="cuda").repeat(2, 1, 1)
            o.step()
        moved = (1 - p.detach().float()).diagonal(dim1=1, dim2=2)
        assert (moved > 0.02).all() if masters else (moved == 0).all()


def test_what_it_refuses_and_leaves_alone(pkg):
    _, _, optim = pkg
    vector = torch.nn.Parameter(torch.zeros(5, device="cuda"))
    with pytest.raises(ValueError):
        optim.Muon([vector])
    with pytest.raises(ValueError):
        optim.Muon([torch.nn.Parameter(torch.zeros((4, 4), device="cuda", dtype=torch.float16))])
    with pytest.raises(ValueError):
        optim.Muon([torch.nn.Parameter(torch.zeros((4, 6), device="cuda").t())])
    with pytest.raises(ValueError):
        optim.Muon([torch.nn.Parameter(torch.zeros((4, 4), device="cuda"))], lr=-1.0)
    p, q = parameters(torch.float32)[:2]
    q.grad = None
    before = q.detach().clone()
    o = optim.Muon([p, q])
    o.step()
    assert torch.equal(q, before) and q not in o.state


def test_gradients_that_are_views(pkg):
    _, _, optim = pkg
    p, q = parameters(torch.float32)[:2]
    q.data.copy_(p.data)
    wide = torch.zeros((4, 48, 41), device="cuda")
    wide[:, :, 1:] = p.grad
    q.grad = wide[:, :, 1:]
    optim.Muon([p]).step()
    optim.Muon([q]).step()
    assert torch.equal(p, q)


def test_the_example_learns(pkg):
    spec = importlib.util.spec_from_file_location("train_lm", os.path.join(ROOT, "examples", "train_lm.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, whole, single, mean = example.train(steps=60, vocab=257, width=64, layers=2, tokens=512, say=None)
    assert torch.isfinite(losses).all()
    assert losses[0].item() > 0.8 * math.log(257) and losses[-5:].mean().item() < 0.5 * losses[0].item()
    assert torch.isfinite(mean) and (whole - single).abs().max().item() <= 1e-4
