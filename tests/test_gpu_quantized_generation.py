"""The 8-bit projections and the 4-bit cache as one model: examples/quantized_generation.py."""
import os
import sys

import pytest

from koala_synth import chain_tree, get_config, predictable_pair, target_weights

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_generation_of_a_predictable_pair():
    """The target's successor of token t is t + 1 by construction, with margins far above what 8 and 4 bits cost; the draft head is right
    some of the time, so that rows are committed from all over the tree."""
    import torch
    import quantized_generation as Q
    cfg = get_config("cfg2_small")
    target, draft = predictable_pair(cfg, 0, sigma=6.0, cache=True)
    for start, n in ((200, 100), (5, 3)):
        prompt = torch.arange(start, start + n, dtype=torch.int32, device="cuda")
        tokens, accepted = Q.generate(cfg, target, draft, prompt, 40)
        assert tokens == [(start + n + i) % cfg["vocab"] for i in range(40)]
        assert 0 < max(accepted) <= cfg["tree_template"].depth


def test_verifying_a_chain_is_decoding_step_by_step():
    """Random weights, one layer: the rows of a chain verified at once against the same tokens one by one, committed each time.  What is
    stored depends on the tokens and positions alone and is the same bit for bit.  Attention rounds to bfloat16 (2^-8 of the value) what
    carries probabilities of 11 bits (2^-12 of the largest value at most, either way of calling it)."""
    import torch
    import quantized_generation as Q
    from paper_2408_08146_amd import packing, tree_masks
    cfg = dict(get_config("cfg2_small"), n_layers=1)
    w = target_weights(cfg, 0, norm_gain="random", cache=True)
    model = Q.QuantizedTarget(cfg, lambda n: packing._dev(w, n, "cuda", "bf16"), 2, 256, page=16)
    g = torch.Generator(device="cuda").manual_seed(1)
    prompt = torch.randint(0, cfg["vocab"], (2, 90), generator=g, device="cuda").int()
    model.prefill(prompt)
    assert model.ctx_len.tolist() == [90, 90]
    tree = chain_tree(7)
    T = len(tree.parent)
    tokens = torch.randint(0, cfg["vocab"], (2, T), generator=g, device="cuda").int()
    b = model.buffers(T)
    b["tokens"].copy_(tokens)
    model.verify(b, torch.arange(T, dtype=torch.int32, device="cuda"), tree_masks(tree))
    heads, dh = cfg["n_heads"], cfg["head_dim"]
    kv = [torch.empty(1, 2, 90 + T, heads, dh, device="cuda") for _ in range(4)]
    model.cache.read(None, None, kv[0], kv[1])
    vmax = kv[1].abs().max()
    one = model.buffers(1)
    for i in range(T):
        one["tokens"].copy_(tokens[:, i:i + 1])
        model.verify(one)
        model.cache.commit(torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 1, dtype=torch.int32, device="cuda"))
        x, y = one["att"][:, 0].float(), b["att"][:, i].float()
        assert ((x - y).abs() <= 2.0 ** -8 * (x.abs() + y.abs()) + 2.0 ** -11 * vmax).all()
    assert model.ctx_len.tolist() == [90 + T] * 2
    model.cache.read(None, None, kv[2], kv[3])
    assert torch.equal(kv[0], kv[2]) and torch.equal(kv[1], kv[3])


def test_a_captured_verification_replays():
    """Every replay against the eager call, the sequence growing in between."""
    import torch
    import quantized_generation as Q
    from paper_2408_08146_amd import packing, tree_masks
    cfg = get_config("cfg2_small")
    w = target_weights(cfg, 0, norm_gain="random", cache=True)
    model = Q.QuantizedTarget(cfg, lambda n: packing._dev(w, n, "cuda", "bf16"), 1, 256)
    tree = cfg["tree_template"]
    depth = [0]
    for p in tree.parent[1:]:
        depth.append(depth[int(p)] + 1)
    depth, mask = torch.tensor(depth, dtype=torch.int32, device="cuda"), tree_masks(tree)
    model.prefill(torch.arange(20, dtype=torch.int32, device="cuda").view(1, -1))
    b, e = model.buffers(tree.n_nodes), model.buffers(tree.n_nodes)
    replay = model.captured(b, depth, mask)
    for i in range(4):
        tokens = torch.randint(0, cfg["vocab"], (1, tree.n_nodes), device="cuda").int()
        b["tokens"].copy_(tokens)
        e["tokens"].copy_(tokens)
        replay()
        torch.cuda.synchronize()
        model.verify(e, depth, mask)
        for name in ("logits", "feat", "greedy"):
            assert torch.equal(b[name], e[name]), (i, name)
        path = torch.tensor([[0, 1, 5]], dtype=torch.int32, device="cuda")
        model.cache.commit(torch.tensor([2], dtype=torch.int32, device="cuda"), path)
    assert model.ctx_len.item() == 32
