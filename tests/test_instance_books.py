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
    return (list(node.free_seqs), dict(node.origin), {k: list(h) for k, h in node.blocks.items()}, {s: t.tolist() for s, t in node.tokens.items()},
            node.cache.books.refs[:], node.cache.books.lengths[:])


def check_books(node):
    m = node.cache.books
    assert sorted(node.free_seqs + list(node.tokens)) == list(range(len(m.lengths)))
    for s, t in node.tokens.items():
        assert m.lengths[s] == len(t) and node.origin[s][1] % m.B == 0
    for s in node.free_seqs:
        assert m.lengths[s] == 0
    assert set(node.origin) == set(node.tokens) and all(h and set(h) <= set(node.tokens) for h in node.blocks.values())


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


def decode_alone(make, tokens, steps, followed):
    """Logits of a sequence run by itself, fed the tokens that were decoded."""
    node = make()
    seqs, logits = node.admit([tokens], room=steps)
    out = [logits[0]]
    for t in followed:
        out.append(node._forward(seqs, [np.asarray([t], dtype=np.uint32)])[0])
    return out


def test_a_reused_id_is_another_origin(make):
    """Children of a sequence, and children of the one that its id went to, decode side by side."""
    import torch
    rng, node = np.random.default_rng(3), make(pages=200, max_seqs=12)
    first, other = prompt(rng, 32), prompt(rng, 32)
    parent, _ = node.admit([prompt(rng, first, 3)])
    old, old_logits = node.admit([prompt(rng, first, 2), prompt(rng, first, 5)], room=3)
    node.drop(parent)
    again, _ = node.admit([prompt(rng, other, 4)])
    assert again == parent   # the id is given out again
    new, new_logits = node.admit([prompt(rng, other, 1), prompt(rng, other, 7)], room=3)
    assert node.reused == 4 * 32
    seqs, logits = old + new, torch.cat([old_logits, new_logits])
    start = [node.tokens[s] for s in seqs]
    decoded = node.decode(seqs, logits, 3)
    assert node.cache.last_error() == 0
    for i, tokens in enumerate(start):
        alone = decode_alone(make, tokens, 3, decoded[:, i].tolist())
        # the same sums in 32 bits in another order: far less than 2^-12 of logits of order 1
        assert [int(x.argmax()) for x in alone[:3]] == decoded[:, i].tolist()
        assert float((logits[i] - alone[0]).abs().max()) < 2.0 ** -12
    offsets, prefixes = node.groups(seqs)
    assert offsets.tolist() == [0, 2, 4] and prefixes.tolist() == [32, 32]
    check_books(node)


@pytest.mark.parametrize("gone", [0, 1, 2])
def test_a_prefix_stays_held_while_someone_holds_it(make, gone):
    """Of three sequences with one prefix any may be dropped: the others' pages are found."""
    rng, node = np.random.default_rng(5), make(pages=200, max_seqs=12)
    head = prompt(rng, 48)
    held = [node.admit([prompt(rng, head, n)])[0][0] for n in (3, 20, 9)]
    assert node.reused == 2 * 48
    node.drop([held[gone]])
    before = node.reused
    seqs, _ = node.admit([prompt(rng, head, 4)])
    assert node.reused - before == 48
    check_books(node)
    node.drop([s for s in held if s in node.tokens and s not in seqs] + seqs)
    assert node.blocks == {} and not any(node.cache.books.refs)
    _, reused = node.admit([prompt(rng, head, 4)]), node.reused
    assert reused == before + 48   # nobody holds it any more


def test_decoding_past_the_pages_is_an_error(make):
    """A step that the pages do not suffice for raises; what is held stays as it was."""
    from paper_2602_06502_gb300 import dualmap as D
    rng, node = np.random.default_rng(6), make(pages=4)
    seqs, logits = node.admit([prompt(rng, 30), prompt(rng, 31)])
    with pytest.raises(D.DualMapError):
        node.decode(seqs, logits, 5)
    assert sorted(len(node.tokens[s]) for s in seqs) == [31, 32]   # one step fitted
    check_books(node)
    assert node.cache.last_error() == 0


def test_a_prompt_that_fails_leaves_nothing(make, monkeypatch):
    from paper_2602_06502_gb300 import dualmap as D
    rng, node = np.random.default_rng(7), make()
    head = prompt(rng, 32)
    node.admit([prompt(rng, head, 3)])
    before = books(node)

    def refused(*a, **k):
        node.cache.error = D.DM_ERR_INVALID_ARG

    with monkeypatch.context() as m:
        m.setattr(node.cache, "plan", refused)
        with pytest.raises(D.DualMapError):
            node.admit([prompt(rng, head, 5), prompt(rng, 12)])
    after = books(node)
    assert sorted(after[0]) == sorted(before[0]) and after[1:] == before[1:] and node.reused == 0
