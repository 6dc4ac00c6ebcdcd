"""The example of decoding by drafted trees: every token it produced is one that the model itself chooses."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("tree_decoding", os.path.join(ROOT, "examples", "tree_decoding.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_tokens_are_the_models_own(example):
    """A plain pass in 64 bits over the whole text: at every position the token that follows has the largest logit, up to the roundings of
    the bf16 path (queries, keys and values, the attended row and the hidden row are each rounded to 8 bits: logits of unit spread
    move by a few times 2^-8; 0.1 is allowed)."""
    model, text = example.run(steps=24, sequences=3, seed=2)
    E, W, O, A, B = (x.cpu().double() for x in (model.embedding, model.qkv, model.out, model.A, model.B))
    hq, hk, D = example.Q_HEADS, example.KV_HEADS, example.HEAD_DIM
    assert text[3] == text[0]                                   # the fork goes on as its parent does
    for t in text:
        assert len(t) > 37 + 24                                 # some drafts were accepted
        x = E[torch.tensor(t)]
        qkv = (x @ W).view(len(t), hq + 2 * hk, D)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk].repeat_interleave(hq // hk, 1), qkv[:, hq + hk:].repeat_interleave(hq // hk, 1)
        s = torch.einsum("thd,shd->hts", q, k) * D ** -0.5
        s = s.masked_fill(torch.ones(len(t), len(t)).triu(1).bool(), -float("inf"))
        h = x + torch.einsum("hts,shd->thd", s.softmax(-1), v).reshape(len(t), -1) @ O
        z = (h @ A) @ B
        for i in range(36, len(t) - 1):
            assert z[i, t[i + 1]] >= z[i].max() - 0.1 * z[i].std(), (i, z[i, t[i + 1]].item(), z[i].max().item())
