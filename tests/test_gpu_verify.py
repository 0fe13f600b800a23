"""Verification of drafted tokens against a plain implementation: decisions
and tokens are whole numbers and have to be equal."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2608_27513_amd import damp as D
from paper_2608_27513_amd import serving as S

pytestmark = pytest.mark.gpu


def case(seed, B, K, V, dtype=torch.float32, noise=0.6):
    gen = torch.Generator().manual_seed(seed)
    x = 2.0 * torch.randn(B, K + 1, V, generator=gen)
    p = torch.softmax(x, -1).to(dtype)
    q = torch.softmax(x[:, :K] + noise * torch.randn(B, K, V, generator=gen), -1).to(dtype)
    race = torch.empty(B, K, V).exponential_(generator=gen)
    tokens = (q.float() / race).argmax(-1).to(torch.int32)
    u = torch.rand(B, K + 1, generator=gen)
    return p, q, tokens, u


def check(p, q, tokens, u, lens=None, ws=None):
    B, K1, V = p.shape
    host = lambda t: t.double().numpy()  # noqa: E731
    n = np.full(B, K1 - 1) if lens is None else np.asarray(lens)
    want_a, want_o = ref.verify(host(p), host(q), tokens.numpy(), host(u), n)
    a, o = S.damp_verify_drafts(p.cuda(), q.cuda(), tokens.cuda(), u.cuda(),
                                lens=None if lens is None else
                                torch.tensor(lens, dtype=torch.int32).cuda(), workspace=ws)
    assert a.tolist() == want_a.tolist()
    assert o.tolist() == want_o.tolist()
    return want_a


@pytest.mark.parametrize("V", [1, 2, 3, 5, 63, 255, 256, 257, 1000, 4095, 4096, 4097, 8191, 8193,
                               32000, 70001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_vocabularies(V, dtype):
    print(f"verify V={V} {dtype}", flush=True)
    got = []
    for seed in range(3):
        got += check(*case(100 * seed + V, 5, 3, V, dtype)).tolist()
    if V >= 255:
        assert 0 < sum(got) < 45  # some drafts stand and some do not


@pytest.mark.parametrize("B,K", [(1, 1), (1, 8), (3, 0), (64, 5), (300, 2), (2, 300), (3001, 1)])
def test_batches(B, K):
    print(f"verify B={B} K={K}", flush=True)
    check(*case(B + K, B, K, 997, noise=0.05))


def test_the_largest_batch():
    """65535 requests: more than have a line of their own for what counts their
    workgroups, several of them each."""
    print("verify B=65535", flush=True)
    B, V = 65535, 300
    p = torch.zeros(B, 1, V, device="cuda")
    at = torch.arange(B, device="cuda") * 7 % V
    p[torch.arange(B, device="cuda"), 0, at] = 0.5
    a, o = S.damp_verify_drafts(p, p[:, :0], torch.zeros(B, 0, dtype=torch.int32, device="cuda"),
                                torch.full((B, 1), 0.3, device="cuda"))
    assert torch.equal(o[:, 0].long(), at) and not bool(a.any())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_requests_of_several_workgroups(dtype):
    """Batches whose requests are each summed by several workgroups, one
    workspace for all of them: the last workgroup of each is found, whichever
    it is, call after call."""
    print(f"verify several workgroups {dtype}", flush=True)
    piece = 256 if dtype is torch.float32 else 512
    # pieces of a row, and workgroups of 4 waves that take ceil(pieces B / 4096) each
    shapes = [(700, 13, 2), (128, 9, 3), (500, 21, 2), (40, 33, 9), (3, 64, 16)]
    ws = torch.zeros(max(S.damp_verify_workspace_bytes(B, piece * n) for B, n, _ in shapes),
                     dtype=torch.uint8, device="cuda")
    for B, n, blocks in shapes:
        steps = -(-n * B // 4096)
        assert -(-n // (4 * steps)) == blocks
        for seed in range(3):
            check(*case(B + seed, B, 1, piece * n - 5 * seed, dtype), ws=ws)
        assert not bool(ws[:1 << 18].any())


def test_lengths():
    """Drafts of every length beside each other; lengths are cut to [0, K]."""
    print("verify lengths", flush=True)
    p, q, tokens, u = case(7, 8, 5, 501, noise=0.1)
    check(p, q, tokens, u, lens=[0, 1, 2, 3, 4, 5, 9, -4])


def test_a_workspace_serves_call_after_call():
    print("verify workspace", flush=True)
    ws = torch.zeros(S.damp_verify_workspace_bytes(6, 20001), dtype=torch.uint8, device="cuda")
    for seed, (B, V) in enumerate([(6, 20001), (1, 20001), (6, 300), (3, 9000), (6, 20001)]):
        check(*case(seed, B, 4, V), ws=ws)
        assert not bool(ws[:1 << 18].any())


def test_drawn_numbers_at_their_ends():
    """u = 0 and the largest below 1 draw the first and the last token with
    weight; numbers outside [0, 1) and NaN are cut."""
    print("verify ends", flush=True)
    V = 9001
    p, q, tokens, u = case(8, 6, 0, V)
    p[:, :, :4] = 0.0
    p[:, :, -3:] = 0.0
    u[:, 0] = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 7.0, -1.0, float("nan")])
    a, o = S.damp_verify_drafts(p.cuda(), q.cuda(), tokens.cuda(), u.cuda())
    check(p, q, tokens, u)
    assert o[0, 0] == 4 and o[4, 0] == 4 and o[5, 0] == 4


def cut(u):
    """Uniform numbers as the definition takes them: in [0, 1 - 2^-24], NaN as 0."""
    return u.nan_to_num(0.0, posinf=1.0, neginf=0.0).clamp(0.0, 1.0 - 2.0 ** -24)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_judging_numbers_at_their_ends(dtype):
    """The numbers that judge drafts are cut like the one that draws: 1 and more
    accept a draft that is as probable as its target, none accepts one that the
    target never makes, NaN and negative ones count as 0."""
    print(f"verify judging ends {dtype}", flush=True)
    ends = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 7.0, float("inf"), -1.0, float("-inf"),
                         float("nan")])
    B, V = len(ends), 600
    p, q, tokens, u = case(15, B, 2, V, dtype)
    rows = torch.arange(B)
    equal, never = q.clone(), p.clone()
    equal[:, 0] = p[:, 0]
    never[rows, 0, tokens[:, 0].long()] = 0.0
    u[:, 0] = ends
    for target, draft, first in ((p, equal, True), (never, q, False)):
        for other in (u[:, 1].clone(), ends.flip(0)):
            now = u.clone()
            now[:, 1] = other
            host = lambda t: t.double().numpy()  # noqa: E731
            want_a, want_o = ref.verify(host(target), host(draft), tokens.numpy(), host(cut(now)),
                                        np.full(B, 2))
            a, o = S.damp_verify_drafts(target.cuda(), draft.cuda(), tokens.cuda(), now.cuda())
            assert a.tolist() == want_a.tolist() and o.tolist() == want_o.tolist()
            assert ((a > 0) == first).all() and bool((o[rows, a.long()] >= 0).all())


def test_one_token_has_all_the_weight():
    print("verify one", flush=True)
    for V, x in ((1, 0), (4096, 4095), (4097, 4096), (12345, 8191), (12345, 8192), (12345, 0)):
        p = torch.zeros(2, 1, V)
        p[:, 0, x] = 1.0
        u = torch.tensor([[0.0], [1.0 - 2.0 ** -24]])
        check(p, torch.zeros(2, 0, V), torch.zeros(2, 0, dtype=torch.int32), u)


def test_rows_without_weight():
    """A row of zeros, of NaN, of negative numbers, or a draft that covers the
    target leaves nothing to draw: the next token is -1."""
    print("verify empty", flush=True)
    V = 5000
    p, q, tokens, u = case(9, 6, 1, V)
    u[:, 0] = 1.0 - 2.0 ** -24
    for b, bad in enumerate([0.0, float("nan"), -1.0, float("-inf")]):
        p[b] = bad
    p[4, 0] = q[4, 0] * 0.5
    q[5, 0, int(tokens[5, 0])] = 1.0
    want = check(p, q, tokens, u)
    assert want[:4].tolist() == [0, 0, 0, 0]


def test_infinities_and_unnormalised_rows():
    print("verify infinities", flush=True)
    V = 4500
    p, q, tokens, u = case(10, 5, 2, V)
    p[0, 0, 17] = float("inf")
    q[1, 0, int(tokens[1, 0])] = float("inf")
    p[2] *= 30.0
    q[3] *= 0.01
    p[4, :, ::2] = float("nan")
    check(p, q, tokens, u)


def test_equal_distributions_accept_every_draft():
    print("verify equal", flush=True)
    p, _, tokens, u = case(11, 16, 6, 3001, noise=0.0)
    assert check(p, p[:, :6].clone(), tokens, u).tolist() == [6] * 16


def test_drafted_tokens_outside_the_vocabulary_never_stand():
    print("verify outside", flush=True)
    p, q, tokens, u = case(12, 4, 3, 700, noise=0.0)
    tokens[0, 1], tokens[1, 0], tokens[2, 2], tokens[3, 0] = 700, -1, 2 ** 31 - 1, -2 ** 31
    assert check(p, q, tokens, u).tolist() == [1, 0, 2, 0]


def test_boundaries_are_exact():
    """u q = p refuses, a hair under stands; thresholds on a weight's edge
    draw the next token."""
    print("verify exact", flush=True)
    V = 64
    p = torch.full((3, 2, V), 1.0 / 64)
    q = torch.full((3, 1, V), 1.0 / 32)
    tokens = torch.full((3, 1), 5, dtype=torch.int32)
    u = torch.tensor([[0.5, 0.5], [0.5 - 2.0 ** -25, 0.25], [0.5 + 2.0 ** -24, 0.0]])
    assert check(p, q, tokens, u).tolist() == [0, 1, 0]
    _, o = S.damp_verify_drafts(p[:, :1].contiguous().cuda(), q[:, :0].contiguous().cuda(),
                                tokens[:, :0].contiguous().cuda(),
                                torch.tensor([[0.5], [0.5 - 2.0 ** -24], [0.25]]).cuda())
    assert o[:, 0].tolist() == [32, 31, 16]


def test_tiny_weights_sum_exactly():
    """Weights of single units of 2^-40 beside large ones: sums do not round."""
    print("verify tiny", flush=True)
    V = 100000
    p = torch.full((2, 1, V), 2.0 ** -40)
    p[1, 0, 50000] = 1.0
    u = torch.tensor([[0.7311], [2.0 ** -24]])
    check(p, torch.zeros(2, 0, V), torch.zeros(2, 0, dtype=torch.int32), u)


def test_offsets_beyond_32_bits():
    """Rows past 2^32 bytes of p and q."""
    print("verify offsets", flush=True)
    B, K, V = 1200, 3, 300000
    p = torch.zeros(B, K + 1, V, device="cuda")  # 5.8 GB
    q = torch.zeros(B, K, V, device="cuda")      # 4.3 GB
    tokens = torch.zeros(B, K, dtype=torch.int32, device="cuda")
    u = torch.full((B, K + 1), 0.5, device="cuda")
    for i in range(K):
        q[:, i, 7 + i] = 1.0
        p[:, i, 7 + i] = 0.75
        p[:, i, V - 2] = 0.25
        tokens[:, i] = 7 + i
    p[:, K, V - 1] = 1.0
    u[B - 1, 2] = 0.9
    a, o = S.damp_verify_drafts(p, q, tokens, u)
    assert a.tolist() == [3] * (B - 1) + [2]
    assert o[:-1].cpu().unique(dim=0).tolist() == [[7, 8, 9, V - 1]]
    assert o[-1].tolist() == [7, 8, V - 2, -1]


def test_graph_replays():
    print("verify graph", flush=True)
    p, q, tokens, u = (t.cuda() for t in case(13, 4, 3, 9000))
    ws = torch.zeros(S.damp_verify_workspace_bytes(4, 9000), dtype=torch.uint8, device="cuda")
    a, o = S.damp_verify_drafts(p, q, tokens, u, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a2, o2 = S.damp_verify_drafts(p, q, tokens, u, workspace=ws)
    for i in range(4):
        if i == 2:
            u.copy_(torch.rand_like(u))
            a, o = S.damp_verify_drafts(p, q, tokens, u, workspace=ws)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, a2) and torch.equal(o, o2), i


def test_binding_refusals():
    p, q, tokens, u = (t.cuda() for t in case(14, 2, 3, 100))
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        S.damp_verify_drafts(p.half(), q.half(), tokens, u)
    with pytest.raises(ValueError, match="q must be"):
        S.damp_verify_drafts(p, q.bfloat16(), tokens, u)
    with pytest.raises(ValueError, match="tokens"):
        S.damp_verify_drafts(p, q, tokens.long(), u)
    with pytest.raises(ValueError, match="u has shape"):
        S.damp_verify_drafts(p, q, tokens, u[:, :3].contiguous())
    with pytest.raises(D.DampError, match="workspace"):
        S.damp_verify_drafts(p, q, tokens, u, workspace=torch.zeros(1, dtype=torch.uint8,
                                                                    device="cuda"))
