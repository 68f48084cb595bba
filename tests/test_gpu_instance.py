"""The instance example: forking from held prefixes and reading them once
gives what running each prompt alone gives, and pages are neither lost nor
shared wrongly."""

import numpy as np
import pytest

from parity_harness import lib_ready

pytestmark = pytest.mark.gpu


def prompts(rng, shapes, vocab):
    """shapes: (prefix name, prefix tokens, own tokens); equal names share tokens."""
    heads = {}
    out = []
    for name, p, own in shapes:
        head = heads.setdefault(name, rng.integers(0, vocab, size=4096).astype(np.uint32))
        out.append(np.concatenate([head[:p], rng.integers(0, vocab, size=own).astype(np.uint32)]))
    return out


def make(pages=600):
    from paper_2602_06502_gb300.instance import Instance
    return Instance(pages=pages, max_tokens=700, max_seqs=40, layers=2, q_heads=8, kv_heads=2, head_dim=64, vocab=500, seed=3)


def test_reused_prefixes_give_the_same_logits():
    lib_ready()
    import torch
    rng = np.random.default_rng(1)
    node, alone = make(), make()
    first = prompts(rng, [("a", 200, 5), ("b", 64, 40)], 500)
    kept, _ = node.admit(first)
    a, b = first[0][:192], first[1][:64]
    later = [np.concatenate([a, rng.integers(0, 500, size=n).astype(np.uint32)]) for n in (1, 30, 7, 200)]
    later += [np.concatenate([b, rng.integers(0, 500, size=n).astype(np.uint32)]) for n in (3, 17)]
    later += prompts(rng, [("c", 20, 3)], 500)
    seqs, logits = node.admit(later)
    assert node.reused >= 4 * 192 + 2 * 64
    tokens = node.decode(seqs, logits, 5)
    assert node.cache.last_error() == 0
    by_tokens = {later[i].tobytes(): i for i in range(len(later))}
    for k, s in enumerate(seqs):
        i = by_tokens[node.tokens[s][:-5].tobytes()]
        got, ref = alone.admit([later[i]])
        # both round activations to bfloat16 at the same places; sums in another order move
        # an activation by a unit in its last place (2^-8) here and there, over two layers
        far = (logits[k].float() - ref[0].float()).norm() / ref[0].float().norm()
        assert float(far) < 2.0 ** -5, (i, float(far))
        alone.drop(got)
        assert tokens.shape == (5, len(seqs))
    assert int(alone.cache.refs.sum()) == 0
    shared = int((node.cache.refs > 0).sum()), int(node.cache.refs.sum())
    assert shared[1] - shared[0] >= 4 * 12 + 2 * 4      # pages that were not stored again
    node.drop(seqs + kept)
    assert int(node.cache.refs.abs().sum()) == 0 and int(node.cache.lengths.sum()) == 0


def test_room_is_made_by_dropping_the_oldest():
    lib_ready()
    rng = np.random.default_rng(2)
    node = make(pages=90)
    for _ in range(8):
        batch = prompts(rng, [("x", 128, 30), ("y", 160, 9), ("z", 0, 100)], 500)
        seqs, logits = node.admit(batch, room=3)
        node.decode(seqs, logits, 3)
        assert node.cache.last_error() == 0
        for s in seqs:
            assert int(node.cache.lengths[s]) == len(node.tokens[s])
        held = sum(-(-len(t) // 16) for t in node.tokens.values())
        assert int(node.cache.refs.sum()) == held


def test_behind_the_router():
    lib_ready()
    from paper_2602_06502_gb300.instance import run
    rows = list(run("tiny", instance=1, batches=2, decode=3, overrides=dict(n_requests=400, batch=200), pages=4096))
    assert len(rows) == 2 and rows[1]["requests"] > 0
    assert 0 < rows[1]["reused_tokens"] <= rows[1]["router_hit_tokens"]
    assert rows[1]["reused_tokens"] + rows[1]["computed_tokens"] == rows[1]["prompt_tokens"] + 3 * rows[1]["requests"]


def test_decoded_steps_give_the_same_logits():
    """Step by step: sequences that decode together behind shared prefixes, and each alone, fed the same tokens."""
    lib_ready()
    rng = np.random.default_rng(4)
    node, alone = make(), make()
    first = prompts(rng, [("a", 200, 5), ("b", 64, 40)], 500)
    node.admit(first)
    batch = [np.concatenate([first[0][:192], rng.integers(0, 500, size=n).astype(np.uint32)]) for n in (7, 1, 40, 16)]
    batch += [np.concatenate([first[1][:64], rng.integers(0, 500, size=n).astype(np.uint32)]) for n in (3, 15)]
    batch += prompts(rng, [("c", 0, 33)], 500)
    steps = 20   # over the ends of pages
    seqs, logits = node.admit(batch, room=steps)
    assert node.reused == 4 * 192 + 2 * 64
    offsets, prefixes = node.groups(seqs)
    assert sorted(prefixes.tolist()) == [0, 64, 192]
    start = [node.tokens[s] for s in seqs]
    feed = rng.integers(0, 500, size=(steps, len(seqs))).astype(np.uint32)
    together = [logits] + [node._forward(seqs, [t[None] for t in row]) for row in feed]
    for k, tokens in enumerate(start):
        own, ref = alone.admit([tokens], room=steps)
        refs = [ref] + [alone._forward(own, [row[k][None]]) for row in feed]
        for i, (x, y) in enumerate(zip(together, refs)):
            # as for the prompts: a unit in an activation's last place (2^-8) here and there, over two layers
            far = (x[k].float() - y[0].float()).norm() / y[0].float().norm()
            assert float(far) < 2.0 ** -5, (k, i, float(far))
        alone.drop(own)
    assert node.cache.last_error() == 0
