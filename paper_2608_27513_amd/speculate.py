"""Speculative decoding of a small linear-attention model through the library's
serving operators, as a server would put them together.

    python -m paper_2608_27513_amd.speculate

The model (random weights) is a stack of linear-attention layers with one decay
a head; its draft is its own first layers. Requests are prefilled as one packed
batch, forked into several samples each, and decoded in rounds: the draft
proposes K tokens on a scratch slot, the target scores them in one prefill that
keeps no state, the verification counts the drafts that stand, and a prefill
over those - the counts stay on the device as its lengths - moves the states
on. Requests that ended are released and the pools compacted.
"""
from __future__ import annotations

import torch

from . import damp as D
from . import serving as S


PADDED = -2  # a slot id of no slot and not the zero state: a request that is not run


class Model:
    """Layers of linear attention with residuals over a tied embedding, and the
    state pool of their requests."""

    def __init__(self, weights, layers: int, slots: int):
        self.w = dict(weights, layers=weights["layers"][:layers])
        self.HV, self.HK, self.d = weights["HV"], weights["HK"], weights["d"]
        self.pool = D.Pool(D.damp_layout_init(self.d, self.d, 0, D.DAMP_STATE_FP32), layers, slots,
                           self.HV)

    def operands(self, layer, x):
        """q, k, v (views of one fused projection) and g of a layer's tokens."""
        w, kq = self.w["layers"][layer], self.HK * self.d
        h = torch.nn.functional.rms_norm(x, x.shape[-1:])
        q, k, v = (h @ w["qkv"]).split([kq, kq, self.HV * self.d], 1)
        unit = lambda t: torch.nn.functional.normalize(t.unflatten(1, (-1, self.d)), dim=-1)  # noqa: E731
        g = -torch.nn.functional.softplus(h @ w["g"] + w["g0"])
        fused = torch.cat([unit(q).flatten(1), unit(k).flatten(1), v], 1).bfloat16()
        q, k, v = fused.split([kq, kq, self.HV * self.d], 1)
        return (q.unflatten(1, (-1, self.d)), k.unflatten(1, (-1, self.d)),
                v.unflatten(1, (-1, self.d)), g)

    def probabilities(self, x):
        return torch.softmax(torch.nn.functional.rms_norm(x, x.shape[-1:]) @ self.w["out"]
                             / self.w["temperature"], -1)

    def step(self, tokens, slot_in, slot_out):
        """One token for each request: the next token's distribution [B, V]."""
        x = self.w["embed"][tokens.long()]
        for n, w in enumerate(self.w["layers"]):
            o = S.damp_linear_update(self.pool, n, slot_in, *self.operands(n, x), slot_out=slot_out)
            x = x + o.flatten(1) @ w["o"]
        return self.probabilities(x)

    def prompt(self, tokens, slot_in, slot_out, seq_start, seq_len, max_len):
        """Packed tokens: the next token's distribution after each [N, V], and
        every layer's operands for a replay."""
        x, kept = self.w["embed"][tokens.long()], []
        for n, w in enumerate(self.w["layers"]):
            kept.append(self.operands(n, x))
            o = S.damp_linear_prefill(self.pool, n, slot_in, *kept[-1], seq_start, seq_len, max_len,
                                      slot_out=slot_out)
            x = x + o.flatten(1) @ w["o"]
        return self.probabilities(x), kept

    def replay(self, kept, slots, seq_start, seq_len, max_len):
        """Moves the states on over the first seq_len tokens of a prompt() call."""
        for n, operands in enumerate(kept):
            S.damp_linear_prefill(self.pool, n, slots, *operands, seq_start, seq_len, max_len)


def random_weights(seed: int, *, layers=4, HV=4, HK=2, d=64, vocab=1000, temperature=1.0,
                   device="cuda"):
    gen = torch.Generator(device=device).manual_seed(seed)
    width = HV * d
    rnd = lambda *s: torch.randn(s, generator=gen, device=device) * s[0] ** -0.5  # noqa: E731
    return dict(HV=HV, HK=HK, d=d, temperature=temperature, embed=rnd(vocab, width) * vocab ** 0.5,
                out=rnd(width, vocab) * 2,
                layers=[dict(qkv=rnd(width, (2 * HK + HV) * d), g=rnd(width, HV), o=rnd(width, width),
                             g0=torch.linspace(-6.0, 0.0, HV, device=device))
                        for _ in range(layers)])


class Server:
    """Requests of one target model and its draft, their slots, and rounds of
    speculation over all of them. How many slots requests hold is known on the
    host too: an id of no slot left (-1) is the zero state to the linear calls,
    so requests that do not fit have to be refused before they are allocated."""

    def __init__(self, weights, *, draft_layers: int, slots: int, drafts: int, seed: int = 0,
                 device="cuda"):
        self.target = Model(weights, len(weights["layers"]), slots)
        self.draft = Model(weights, draft_layers, slots)
        self.K, self.dev = drafts, device
        self.slots, self.held = slots, 0
        self.refs = torch.zeros(slots, dtype=torch.int32, device=device)
        self.gen = torch.Generator(device=device).manual_seed(seed)
        vocab = weights["embed"].shape[0]
        self.ws = torch.zeros(S.damp_verify_workspace_bytes(slots, vocab), dtype=torch.uint8,
                              device=device)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.gen, device=self.dev)

    def sample(self, p):
        """One token from each row of p [B, V]."""
        B, V = p.shape
        _, out = S.damp_verify_drafts(p[:, None], p.new_empty(B, 0, V),
                                      torch.empty(B, 0, dtype=torch.int32, device=p.device),
                                      self.uniform(B, 1), workspace=self.ws)
        return out[:, 0]

    def admit(self, prompts, samples: int):
        """Prefills the prompts (host lists) together and forks each into
        `samples` requests; returns (slots, pending tokens) of all of them.
        Raises ValueError where they, or the scratch slots that a round of
        drafts takes for each request, would not fit."""
        if samples < 1 or not all(prompts):
            raise ValueError("needs at least one sample, and a token in every prompt")
        held = self.held + len(prompts) * samples
        if held * (2 if self.K else 1) > self.slots:
            raise ValueError(f"{held} requests{' with a scratch slot each' if self.K else ''} "
                             f"do not fit {self.slots} slots")
        self.held = held
        lens = [len(x) - 1 for x in prompts]  # the last token is the first to be stepped
        starts = [sum(lens[:i]) for i in range(len(lens))]
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=self.dev)  # noqa: E731
        tokens = i32([t for x in prompts for t in x[:-1]])
        slots = S.damp_slots_alloc(self.refs, len(prompts) * samples).view(len(prompts), samples)
        first = slots[:, 0].contiguous()
        new = torch.full_like(first, S.DAMP_SLOT_ZERO)
        for m in (self.target, self.draft):
            m.prompt(tokens, new, first, i32(starts), i32(lens), max(lens))
            if samples > 1:
                S.damp_slots_fork(m.pool, first, slots[:, 1:].contiguous())
        return slots.reshape(-1), i32([x[-1] for x in prompts]).repeat_interleave(samples)

    def round(self, slots, pending):
        """K drafts, their verification and the states moved on; returns
        (accepted [B], tokens [B, K + 1], pending). A next token of -1 (no token
        had weight) ends its request: from the next round on it takes part as a
        padded one, with -1 accepted, tokens of -1 and its state left alone."""
        B, K = slots.numel(), self.K
        live = pending >= 0
        slots = torch.where(live, slots, PADDED)
        scratch = S.damp_slots_alloc(self.refs, B if K else 0)
        from_scratch = torch.where(live, scratch, PADDED) if K else scratch
        tokens, dists = [pending], []
        for i in range(K):
            q = self.draft.step(tokens[-1], slots if i == 0 else from_scratch, scratch)
            tokens.append(self.sample(q))
            dists.append(q)
        S.damp_slots_release(self.refs, scratch)
        run = torch.stack(tokens, 1)  # [B, K + 1]
        flat = run.reshape(-1)
        start = torch.arange(0, B * (K + 1), K + 1, dtype=torch.int32, device=self.dev)
        whole = torch.full((B,), K + 1, dtype=torch.int32, device=self.dev)
        unkept = torch.full_like(slots, S.DAMP_SLOT_ZERO)
        p, kept = self.target.prompt(flat, slots, unkept, start, whole, K + 1)
        q = torch.stack(dists, 1) if K else p.new_empty(B, 0, p.shape[1])
        accepted, out = S.damp_verify_drafts(p.view(B, K + 1, -1), q, run[:, 1:].contiguous(),
                                             self.uniform(B, K + 1), workspace=self.ws)
        accepted = torch.where(live, accepted, -1)
        out = torch.where(live[:, None], out, -1)
        stands = accepted + 1
        self.target.replay(kept, slots, start, stands, K + 1)
        self.draft.prompt(flat, slots, slots, start, stands, K + 1)
        return accepted, out, out.gather(1, accepted[:, None].clamp(min=0).long())[:, 0]

    def end(self, slots, ended):
        """Releases the requests at the indices `ended`, compacts both pools and
        returns the others' slots."""
        S.damp_slots_release(self.refs, slots[ended].contiguous())
        again = self.refs.clone()
        where, _ = S.damp_slots_compact(self.target.pool, self.refs)
        S.damp_slots_compact(self.draft.pool, again)
        keep = torch.ones(slots.numel(), dtype=torch.bool, device=self.dev)
        keep[ended] = False
        self.held -= int((~keep).sum())
        return where[slots[keep].long()], keep


def main() -> None:
    weights = random_weights(0)
    server = Server(weights, draft_layers=2, slots=64, drafts=4)
    gen = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, 1000, (n,), generator=gen).tolist() for n in (37, 300, 5, 1024)]
    slots, pending = server.admit(prompts, samples=3)
    made = 0
    for turn in range(16):
        accepted, _, pending = server.round(slots, pending)
        made += int((accepted + 1).sum())
        if turn == 7:  # the second prompt's samples end
            slots, keep = server.end(slots, torch.arange(3, 6, device=slots.device))
            pending = pending[keep].contiguous()
        print(f"round {turn}: {slots.numel()} requests in slots up to {int(slots.max())}, "
              f"{accepted.float().mean():.2f} of {server.K} drafts stand", flush=True)
    print(f"{made} tokens")


if __name__ == "__main__":
    main()
