"""The example program of train_heads.py: a head's output and every gradient against fp64 from the definitions (the oracle), and a
run whose loss falls."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import operators_oracle as oo
from paper_2407_01445_amd import binding as fc
from paper_2407_01445_amd.train_heads import Head, HeadTrainer, features

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().double().cpu().numpy()


def near(got, want, what, tol=2e-2):
    """The chain rounds its activations and gradients to bf16 (2^-8 each) five times over; their errors add up like those of a
    random walk over rows and layers: 2e-2 of the largest value."""
    got, want = f64(got).reshape(want.shape), np.asarray(want)
    assert np.max(np.abs(got - want)) <= tol * np.max(np.abs(want)), (what, np.max(np.abs(got - want)) / np.max(np.abs(want)))


@pytest.mark.parametrize("rows,d,hidden", [(128, 64, 256), (777, 136, 72)])
def test_head_forward_and_gradients(rows, d, hidden):
    head = Head(rows, d, hidden, seed=3)
    rng = np.random.default_rng(rows)
    for k in ("gamma", "beta", "b1", "b2"):
        head.params[k].add_(torch.from_numpy(rng.normal(0, 0.2, head.params[k].shape).astype(np.float32)).cuda())
    x = torch.from_numpy(rng.normal(0.5, 1, (rows, d)).astype(np.float32)).cuda().bfloat16()
    de = torch.from_numpy(rng.normal(0, 1e-2, (rows, d)).astype(np.float32)).cuda().bfloat16()
    e = head.forward(x)
    head.backward(de)
    torch.cuda.synchronize()
    p = {k: f64(v) for k, v in head.params.items()}
    w1, w2 = f64(head.bf16["w1"]), f64(head.bf16["w2"])
    h, mean, rstd = oo.layer_norm(f64(x), p["gamma"], p["beta"], 1e-5)
    z, pre = oo.linear(h, w1, p["b1"], "gelu")
    near(e, oo.linear(z, w2, p["b2"], "", h)[0], "e")
    dw2, db2 = oo.linear_grad_weight(f64(de), z)
    dpre = oo.linear_grad_input(f64(de), w2, pre, "gelu")
    dw1, db1 = oo.linear_grad_weight(dpre, h)
    dx, dgamma, dbeta = oo.layer_norm_grad(f64(x), oo.linear_grad_input(dpre, w1) + f64(de), mean, rstd, p["gamma"])
    for k, want in dict(w2=dw2, b2=db2, w1=dw1, b1=db1, gamma=dgamma, beta=dbeta).items():
        near(head.grads[k], want, k)
    near(head.dx, dx, "dx")


@pytest.mark.parametrize("state_bits", [8, 32])
def test_training_lowers_the_loss_and_keeps_the_copies(state_bits):
    pairs, d = 256, 128
    trainer = HeadTrainer(pairs, d, 256, samples=2 * pairs, state_bits=state_bits, lr=2e-3)
    sets = [features(pairs, d, 0.3, seed) for seed in range(2)]
    losses = []
    for s in range(60):
        k = s % 2
        trainer.step(*sets[k], torch.arange(k * pairs, (k + 1) * pairs, device="cuda"))
        losses.append(float(trainer.loss))
    assert all(np.isfinite(losses)) and losses[-1] < losses[1] - 0.05 * abs(losses[1]), (losses[:4], losses[-4:])
    for head in (trainer.img, trainer.txt):
        for k, copy in head.bf16.items():
            assert torch.equal(copy, head.params[k].bfloat16())


def test_example_runs_as_a_program(capsys, monkeypatch):
    from paper_2407_01445_amd import train_heads
    monkeypatch.setattr("sys.argv", ["train_heads", "--pairs", "64", "--width", "32", "--hidden", "64", "--steps", "3"])
    train_heads.main()
    assert "step 2: loss" in capsys.readouterr().out
