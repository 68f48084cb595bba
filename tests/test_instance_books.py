"""The instance example's bookkeeping, on a cache on the CPU: sequence ids,
room, held prefixes, groups."""

import numpy as np
import pytest


@pytest.fixture
def make(monkeypatch):
    import torch

    from cpu_cache import CpuCache
    from paper_2602_06502_gb300 import instance
    monkeypatch.setattr(instance, "PagedCache", CpuCache)

    def build(pages=60, max_seqs=6, max_tokens=200):
        return instance.Instance(pages=pages, max_tokens=max_tokens, max_seqs=max_seqs, layers=2, q_heads=4, kv_heads=2, head_dim=16,
                                 vocab=50, dtype=torch.float32, seed=4, device="cpu")
    return build


def prompt(rng, *parts):
    """Token arrays, and numbers of random tokens."""
    return np.concatenate([x if isinstance(x, np.ndarray) else rng.integers(0, 50, size=x) for x in parts]).astype(np.uint32)


def books(node):
    return (list(node.free_seqs), dict(node.origin), dict(node.blocks), {s: t.tolist() for s, t in node.tokens.items()},
            node.cache.books.refs[:], node.cache.books.lengths[:])


def check_books(node):
    m = node.cache.books
    assert sorted(node.free_seqs + list(node.tokens)) == list(range(len(m.lengths)))
    for s, t in node.tokens.items():
        assert m.lengths[s] == len(t) and node.origin[s][1] % m.B == 0
    for s in node.free_seqs:
        assert m.lengths[s] == 0
    assert set(node.origin) == set(node.tokens) and set(node.blocks.values()) <= set(node.tokens)


def test_oldest_sequences_make_room_for_ids(make):
    """More admissions than there are ids, with pages to spare."""
    rng, node = np.random.default_rng(1), make(pages=400, max_seqs=5)
    held = []
    for _ in range(6):
        seqs, logits = node.admit([prompt(rng, 20), prompt(rng, 30)])
        held += [node.tokens[s].tolist() for s in seqs]
        assert bool(logits.isfinite().all()) and len(node.tokens) <= 5
        check_books(node)
    # the youngest are the ones that are held
    assert sorted(t.tolist() for t in node.tokens.values()) == sorted(held[-len(node.tokens):])


@pytest.mark.parametrize("batch,room", [((10,) * 7, 0),              # more prompts than ids
                                        ((150, 150, 150), 0),        # more pages than there are
                                        ((150, 130), 30),            # with the tokens to be decoded
                                        ((20, 190), 20),             # longer than a sequence can be
                                        ((20, 0), 5)])               # no tokens
def test_a_batch_that_cannot_run_changes_nothing(make, batch, room):
    rng, node = np.random.default_rng(2), make(pages=18, max_seqs=6)
    node.admit([prompt(rng, 40), prompt(rng, 17)])
    before = books(node)
    with pytest.raises(ValueError):
        node.admit([prompt(rng, n) for n in batch], room=room)
    assert books(node) == before
    node.admit([prompt(rng, 40)], room=1)
    check_books(node)
