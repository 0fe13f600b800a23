"""The speculative example: the serving operators as they are used together."""
import pytest
import torch

from paper_2608_27513_amd import serving as S
from paper_2608_27513_amd import speculate as X

pytestmark = pytest.mark.gpu


def prompts(lens, vocab, seed=3):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randint(0, vocab, (n,), generator=gen).tolist() for n in lens]


def generate(server, made, rounds):
    """Texts [B] of `rounds` rounds over admitted requests."""
    slots, pending = made
    texts = [[int(t)] for t in pending]
    for _ in range(rounds):
        accepted, out, pending = server.round(slots, pending)
        for b, (a, row) in enumerate(zip(accepted.tolist(), out.tolist())):
            texts[b] += row[:a + 1]
    return texts


def test_greedy_speculation_makes_the_text_of_plain_decoding():
    """At a temperature that leaves one token all the weight, drafts change how
    fast the text comes and nothing of it."""
    print("speculate greedy", flush=True)
    w = X.random_weights(5, vocab=300, temperature=1e-4)
    ps = prompts([20, 3, 150], 300)
    texts = {}
    for K, layers in ((0, 1), (3, 2), (5, 4)):
        server = X.Server(w, draft_layers=layers, slots=16, drafts=K)
        texts[K] = generate(server, server.admit(ps, 1), 24 if K == 0 else 12)
    for K in (3, 5):
        for a, b in zip(texts[0], texts[K]):
            n = min(len(a), len(b), 20)
            assert n >= 13 and a[:n] == b[:n], K


def test_a_draft_equal_to_its_target_stands():
    print("speculate equal", flush=True)
    w = X.random_weights(6, vocab=500)
    server = X.Server(w, draft_layers=4, slots=32, drafts=4)
    slots, pending = server.admit(prompts([10, 70], 500), 4)
    stood = 0
    for _ in range(6):
        accepted, out, pending = server.round(slots, pending)
        stood += int(accepted.sum())
        assert bool((out[:, 0] >= 0).all())
    # p and q differ by roundings of bf16 operands at most: a draft is refused
    # with the probability of the part that those move
    assert stood >= 0.97 * 6 * 8 * 4


def test_states_after_rounds_are_those_of_the_text():
    """Every slot's state equals a prefill of its whole text from nothing:
    forks, replays of the accepted tokens and compaction leave nothing behind."""
    print("speculate states", flush=True)
    w = X.random_weights(7, vocab=400)
    server = X.Server(w, draft_layers=2, slots=24, drafts=3)
    ps = prompts([33, 130, 2], 400)
    slots, pending = server.admit(ps, 2)
    owners = [p for p in ps for _ in range(2)]
    texts = [list(p) for p in owners]
    for turn in range(8):
        accepted, out, pending = server.round(slots, pending)
        for b, (a, row) in enumerate(zip(accepted.tolist(), out.tolist())):
            texts[b] += row[:a + 1]
        if turn == 3:
            slots, keep = server.end(slots, torch.tensor([0, 3], device="cuda"))
            pending = pending[keep].contiguous()
            texts = [t for t, k in zip(texts, keep.tolist()) if k]
            assert sorted(slots.tolist()) == list(range(4))
            assert server.refs.tolist() == [1] * 4 + [0] * 20
    assert server.refs.sum() == 4
    for m in (server.target, server.draft):
        fresh = X.Model(w, len(m.w["layers"]), 24)
        lens = [len(t) - 1 for t in texts]  # the pending token is not in the state yet
        i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
        fresh.prompt(i32([t for x in texts for t in x[:-1]]), torch.full_like(slots, S.DAMP_SLOT_ZERO),
                     slots, i32([sum(lens[:i]) for i in range(4)]), i32(lens), max(lens))
        shape = (len(m.w["layers"]), 24, 4, 64, 64)
        a, b = (x.pool.buffer.view(torch.float32).view(shape)[:, slots.long()] for x in (m, fresh))
        # operands are rounded to bf16 (2^-8) after products whose own rounding
        # depends on the batch: a few of them round the other way
        assert float((a - b).norm() / b.norm()) <= 2.0 ** -8


def test_requests_that_do_not_fit_are_refused():
    """Nothing is allocated for them; what fits, with a scratch slot for each
    request, runs, also after others have ended."""
    print("speculate full", flush=True)
    w = X.random_weights(8, vocab=200)
    server = X.Server(w, draft_layers=2, slots=9, drafts=2)
    ps = prompts([5, 9, 3], 200)
    for bad in ((ps, 2), (ps[:1], 5), ([[]], 1), (ps, 0)):
        with pytest.raises(ValueError):
            server.admit(*bad)
    assert server.refs.tolist() == [0] * 9
    slots, pending = server.admit(ps[:2], 2)
    assert (slots >= 0).all()
    with pytest.raises(ValueError, match="9 slots"):
        server.admit(ps[2:], 1)
    assert int(server.refs.sum()) == 4
    _, _, pending = server.round(slots, pending)
    slots, keep = server.end(slots, torch.tensor([1, 2], device="cuda"))
    more, again = server.admit(ps[2:], 2)
    assert sorted(slots.tolist() + more.tolist()) == [0, 1, 2, 3]
    server.round(torch.cat([slots, more]), torch.cat([pending[keep], again]))
    assert int(server.refs.sum()) == 4
    with pytest.raises(ValueError):
        server.admit(ps[:1], 1)
    whole = X.Server(w, draft_layers=1, slots=3, drafts=0)  # no drafts: no scratch
    slots, pending = whole.admit(ps, 1)
    whole.round(slots, pending)
    with pytest.raises(ValueError, match="4 requests do not fit 3 slots"):
        whole.admit(ps[:1], 1)


def test_a_request_without_a_next_token_ends():
    """A next token of -1 is no token: its request stands still from then on,
    the others go on."""
    print("speculate end", flush=True)
    w = X.random_weights(9, vocab=200)
    server = X.Server(w, draft_layers=2, slots=8, drafts=3)
    slots, pending = server.admit(prompts([5, 9, 3], 200), 1)

    def states(slot):
        return [m.pool.buffer.view(len(m.w["layers"]), 8, -1)[:, slot].clone()
                for m in (server.target, server.draft)]

    ended, live = int(slots[1]), int(slots[0])
    pending[1] = -1
    before, running = states(ended), states(live)
    for _ in range(2):
        accepted, out, pending = server.round(slots, pending)
        assert accepted.tolist()[1] == -1 and out[1].tolist() == [-1] * 4 and int(pending[1]) == -1
        assert (accepted[[0, 2]] >= 0).all() and (pending[[0, 2]] >= 0).all()
    assert all(torch.equal(a, b) for a, b in zip(before, states(ended)))
    assert not any(torch.equal(a, b) for a, b in zip(running, states(live)))
    server.target.w["out"] = torch.full_like(w["out"], float("nan"))  # no token has weight
    accepted, out, pending = server.round(slots, pending)
    assert accepted.tolist() == [0, -1, 0] and pending.tolist() == [-1] * 3
    before = states(live)
    accepted, _, pending = server.round(slots, pending)
    assert accepted.tolist() == [-1] * 3 and pending.tolist() == [-1] * 3
    assert all(torch.equal(a, b) for a, b in zip(before, states(live)))


def test_main_runs(capsys):
    X.main()
    assert "tokens" in capsys.readouterr().out
