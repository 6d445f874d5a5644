"""The example: training in MXFP4 with clipped AdamW falls to the data's entropy, and a token served by
itself has the logits it has in a batch."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_training_and_serving():
    from paper_2603_18112_gb300 import build, mx
    build.build()
    spec = importlib.util.spec_from_file_location("train_mxfp4", os.path.join(ROOT, "examples", "train_mxfp4.py"))
    M = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(M)
    model, copies, losses, floor, step = M.train(steps=150, width=128, vocab=256, batch=2048, log=None)
    assert step.steps.tolist() == [150, 0]
    # of what there is to learn, more than half was learnt
    assert sum(losses[-10:]) / 10 - floor < 0.5 * (losses[0] - floor)
    for p, c in zip(model.params(), copies):
        assert torch.equal(c, p.detach().to(torch.bfloat16))
    # a token's row of every product is the same by itself and in a batch, up to the order of fp32 sums,
    # which may move a bf16 result to its neighbour and what follows by as much
    tokens = torch.arange(24, device="cuda")
    batch = model.forward(tokens, copies[0]).detach().float()
    one = M.serve(model, copies[0], tokens.tolist()).float()
    assert (batch - one).norm() <= 2.0 ** -6 * batch.norm()
    assert mx.tula_mx_error() == 0
