"""The block-decoding example: its operators together, against a plain forward pass in 64 bits over
the values that its cache holds."""
import importlib.util
import math
import os

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example(fd):
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "cached_block_decoding.py")
    spec = importlib.util.spec_from_file_location("cached_block_decoding", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain(example, model, prefix, tokens, first):
    """`forward` in fp64 on the CPU."""
    B, n = tokens.shape
    norm = lambda y: y / torch.sqrt((y * y).mean(-1, keepdim=True) + example.EPS)
    x = model.embed.cpu().double()[tokens.cpu().long()]
    at = torch.arange(first, first + n).repeat(B)
    for layer, cache in zip(model.layers, prefix.caches):
        w = {name: t.cpu().double() for name, t in layer.items()}
        qkv = (norm(x) @ w["qkv"].t()).view(B * n, -1, model.head_dim)
        turn = lambda y, weight: ref.rope(y, weight, at, None, model.inv_freq, example.EPS, False)
        q = turn(qkv[:, :model.heads], w["q_norm"]).view(B, n, model.heads, -1)
        k = turn(qkv[:, model.heads:-model.kv_heads], w["k_norm"]).view(B, n, model.kv_heads, -1)
        v = qkv[:, -model.kv_heads:].reshape(B, n, model.kv_heads, -1)
        out = ref.attention(q, cache, prefix.table.cpu(), prefix.lens.tolist(), k, v)[0]
        x = x + out.flatten(2) @ w["out"].t()
        y = norm(x) @ w["up"].t()
        x = x + (y * torch.sigmoid(y)) @ w["down"].t()
    return norm(x)


def test_forward_over_the_cache(example, monkeypatch):
    """Two layers round their streams and products to bfloat16 some ten times each, at 2^-9 of
    values of order one: the root mean square error stays below 2^-5 of the result's."""
    monkeypatch.setitem(ref.EPS, torch.float64, 0.0)
    model = example.Model(seed=3)
    g = torch.Generator().manual_seed(4)
    prompt = torch.randint(0, model.mask_token, (2, 45), generator=g).int().cuda()
    prefix = example.PrefixCache(model, 2, 80)
    _, state = example.forward(model, prefix, prompt, 0)
    prefix.append(state)
    block = torch.full((2, 7), model.mask_token, dtype=torch.int32, device="cuda")
    block[:, 2] = 5
    got = example.forward(model, prefix, block, 45)[0].cpu().double()
    want = plain(example, model, prefix, block, 45)
    error = float(((got - want) ** 2).mean().sqrt() / (want ** 2).mean().sqrt())
    assert error <= 2.0 ** -5, error


def test_decoding(example):
    model = example.Model(seed=5)
    g = torch.Generator().manual_seed(6)
    prompt = torch.randint(0, model.mask_token, (3, 61), generator=g).int().cuda()
    tokens, steps, prefix = example.decode(model, prompt, 70, block=16, budget=96)
    assert tuple(tokens.shape) == (3, 70) and bool(((tokens >= 0) & (tokens < 1024)).all())
    assert 5 <= steps <= 70 and prefix.lens.tolist() == [96] * 3
    for w in prefix.weights:  # what is held behind the kept keys is nothing
        assert bool(torch.isfinite(w).all()) and bool((w[:, :, 96:] == 0).all())
        assert bool((w >= 0).all()) and math.isfinite(float(w.sum()))
    again = example.decode(model, prompt, 70, block=16, budget=96)
    assert torch.equal(tokens, again[0]) and steps == again[1]
    for a, b in zip(prefix.weights, again[2].weights):
        assert torch.equal(a, b)


def test_without_eviction_nothing_is_lost(example):
    model = example.Model(layers=1, seed=7)
    prompt = torch.arange(40, dtype=torch.int32).view(1, 40).cuda()
    tokens, _, prefix = example.decode(model, prompt, 33, block=32, budget=500)
    assert tuple(tokens.shape) == (1, 33) and prefix.lens.tolist() == [73]
    total = float(prefix.weights[0].double().sum())
    # queries of two blocks look at 40 and then 72 cached keys, some of their weight at their own
    assert 0 < total < 33 * model.heads
