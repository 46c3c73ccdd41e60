"""The example that trains a layer and serves it runs, learns, and serves the same tokens with drafts as without."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import gdn_grad

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "train_and_serve.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_and_serve", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.fixture(scope="module")
def trained(example):
    torch.manual_seed(1)
    model = example.Model().cuda()
    return model, example.train(model, 60, np.random.default_rng(1), log=lambda s: None)


def test_training_learns(example, trained):
    losses = trained[1]
    assert losses[0] > 0.9 * np.log(example.V)                 # knows nothing at first
    assert np.mean(losses[-5:]) < 0.75 * losses[0]


def test_the_function_has_the_formulas_gradient(example):
    """fp32 inputs: 1e-5 of each gradient's RMS, the bound of the call's own tests."""
    e, rng = example, np.random.default_rng(2)
    start = torch.tensor([0, 70, 70, 100], dtype=torch.int32, device="cuda")
    sizes = [(e.Hk, e.D), (e.Hk, e.D), (e.Hv, e.D), (e.Hv,), (e.Hv,)]
    x = [np.float32(rng.standard_normal((100,) + s) * (e.D ** -0.5 if i < 2 else 1.0)) for i, s in enumerate(sizes)]
    x[3], x[4] = -np.abs(x[3]) * np.float32(0.1), np.float32(1.0) / (1.0 + np.exp(-x[4]))
    w = np.float32(rng.standard_normal((100, e.Hv, e.D)))
    t = [torch.tensor(y, device="cuda", requires_grad=True) for y in x]
    (e.Scan.apply(*t, start) * torch.tensor(w, device="cuda")).sum().backward()
    for lo, hi in ((0, 70), (70, 100)):
        zero = np.zeros((e.Hv, e.D, e.D))
        want = gdn_grad.backward(zero, *(y[lo:hi] for y in x), e.SCALE, w[lo:hi], zero)
        for got, y in zip(t, want):
            assert np.abs(got.grad[lo:hi].cpu().numpy() - y).max() < 1e-5 * np.sqrt(np.mean(y ** 2))


def test_drafts_change_nothing_but_the_number_of_rounds(example, trained):
    """At temperature 0 a request's tokens are the target's best ones, with four drafts a round or one."""
    rng = np.random.default_rng(3)
    prompts = [example.phrases(rng, [n]) for n in (2, 30, 64, 65, 150)]
    few, gained = example.serve(trained[0], prompts, 4, 6)
    one, _ = example.serve(trained[0], prompts, 1, 30)
    assert all(1.0 <= x <= 5.0 for x in gained) and max(gained) > 1.0
    for a, b, p in zip(few, one, prompts):
        n = min(len(a), len(b))
        assert len(a) >= len(p) + 6 and a[:n] == b[:n]
