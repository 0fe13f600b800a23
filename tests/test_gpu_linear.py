"""Linear attention with one decay a head (prompts and single tokens) against
the recurrence in 64 bits.

Tolerances. Operands are bf16 values and every product of the kernels is good
to fp32's 24 bits, sums are fp32. Results are sums of terms of random sign, in
which the roundings (2^-25 of a partial sum on average) of at most a few
hundred additions meet: about 2^-25 sqrt(500) = 0.7e-6 of the result's norm.
FP32 = 2e-6 leaves a factor of three, and is under what operands cut to 16
bits in two parts would leave (2.8e-6). A bf16 output is off by at most half a
step beside that: bf16 has 8 significant bits, so 2^-8 of its value.
"""
import ctypes

import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2608_27513_amd import damp as D
from paper_2608_27513_amd import serving as S

pytestmark = pytest.mark.gpu

FP32 = 2e-6


def rel(x, y):
    x, y = x.double().cpu(), y.double().cpu()
    return float((x - y).norm() / max(float(y.norm()), 1e-300))


def check_o(o, want, where=None):
    got, want = o.double().cpu(), want.double().cpu()
    if o.dtype is torch.bfloat16:
        rms = float(want.square().mean().sqrt())
        assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() * 1.001 + 10 * FP32 * rms).all()), where
    else:
        assert rel(got, want) <= FP32, where


class Setup:
    """Operands on the CPU and the GPU, and a pool with known states."""

    def __init__(self, seed, n, HV, HK, dk, dv, slots, *, const=False, decay=None, fused=False):
        gen = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=gen)  # noqa: E731
        unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
        self.n, self.HV, self.HK, self.dk, self.dv = n, HV, HK, dk, dv
        wide = torch.cat([unit(rnd(n, HK, dk)).flatten(1), unit(rnd(n, HK, dk)).flatten(1),
                          rnd(n, HV, dv).flatten(1)], 1).bfloat16()
        cut = [0, HK * dk, 2 * HK * dk, 2 * HK * dk + HV * dv]
        shape = [(n, HK, dk), (n, HK, dk), (n, HV, dv)]
        self.cpu = [wide[:, a:b].reshape(s) for a, b, s in zip(cut, cut[1:], shape)]
        if fused:
            dev = wide.cuda()
            self.dev = [dev[:, a:b].unflatten(1, s[1:]) for a, b, s in zip(cut, cut[1:], shape)]
        else:
            self.dev = [x.contiguous().cuda() for x in self.cpu]
        mu = torch.linspace(-6.0, 0.5, HV)
        self.g = -torch.nn.functional.softplus(mu if const else mu + rnd(n, HV))
        if decay is not None:
            self.g = decay(self.g)
        self.state = rnd(slots, HV, dk, dv)
        self.buffer = self.state.cuda().view(torch.uint8).reshape(-1)
        self.now = self.buffer.view(torch.float32).view(slots, HV, dk, dv)
        self.pool = D.Pool(D.damp_layout_init(dk, dv, 0, D.DAMP_STATE_FP32), 1, slots, HV,
                           buffer=self.buffer)
        self.scale = dk ** -0.5

    def want(self, start, length, slot):
        q, k, v = (x[start:start + length] for x in self.cpu)
        g = self.g.expand(self.n, self.HV)[start:start + length]
        S0 = self.state[slot] if slot >= 0 else torch.zeros_like(self.state[0])
        return ref.linear(q, k, v, g, S0, self.scale)


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


SIZES = [(128, 128), (64, 64), (128, 64), (96, 96), (16, 16), (8, 8), (24, 40), (32, 128),
         (256, 256), (200, 136)]


# ------------------------------------------------------------ single tokens

@pytest.mark.parametrize("dk,dv", SIZES)
@pytest.mark.parametrize("o_type", [torch.float32, torch.bfloat16])
def test_update_sizes(dk, dv, o_type):
    print(f"update {dk}x{dv} {o_type}", flush=True)
    for seed, (B, HV, HK) in enumerate([(1, 4, 4), (3, 6, 2), (17, 3, 1)]):
        x = Setup(seed, B, HV, HK, dk, dv, 2 * B + 1, fused=seed == 1, const=seed == 2)
        slots = np.random.RandomState(seed).permutation(2 * B + 1)[:B]
        o = torch.full((B, HV, dv), 7.0, dtype=o_type, device="cuda")
        S.damp_linear_update(x.pool, 0, i32(slots), *x.dev, x.g.cuda(), scale=x.scale, o=o)
        keep = x.state.clone()
        wants = [x.want(b, 1, s) for b, s in enumerate(slots)]
        for s, (_, S1) in zip(slots, wants):
            keep[s] = S1.float()
        check_o(o, torch.cat([w for w, _ in wants]), (dk, dv, seed))
        assert rel(x.now, keep) <= FP32
        untouched = [s for s in range(2 * B + 1) if s not in slots]
        assert torch.equal(x.now[untouched].cpu(), x.state[untouched])


@pytest.mark.parametrize("B,HV,dv", [(1, 32, 128), (2, 32, 128), (7, 32, 128), (40, 32, 128),
                                     (300, 8, 64), (1, 1, 8), (70, 32, 256)])
def test_update_batches(B, HV, dv):
    """Launch shapes from one workgroup to several rounds of the device."""
    print(f"update batch {B} {HV} {dv}", flush=True)
    x = Setup(B, B, HV, 1, 64, dv, B)
    o = S.damp_linear_update(x.pool, 0, i32(list(range(B))), *x.dev, x.g.cuda(), scale=x.scale)
    k, v, a = x.cpu[1].double(), x.cpu[2].double(), x.g.double().exp()
    want = a[..., None, None] * x.state + k[..., None] * v[:, :, None]
    assert rel(x.now, want) <= FP32
    check_o(o, x.scale * (x.cpu[0].double()[..., None] * want).sum(2))


def test_update_slots():
    """Zero states, padded requests, states that are not kept, one state
    continued by several requests, and another target than the source."""
    print("update slots", flush=True)
    x = Setup(5, 8, 4, 2, 64, 48, 9)
    slot_in = [3, 3, -1, -2, 9, 0, -1, 1]
    slot_out = [4, 5, 6, 7, 8, -1, 100, 1]
    o = torch.full((8, 4, 48), 7.0, device="cuda")
    S.damp_linear_update(x.pool, 0, i32(slot_in), *x.dev, x.g.cuda(), slot_out=i32(slot_out),
                         scale=x.scale, o=o)
    state = x.state.clone()
    for b, (a, c) in enumerate(zip(slot_in, slot_out)):
        if a < -1 or a >= 9:
            assert bool((o[b] == 0).all())
            continue
        w, S1 = x.want(b, 1, a)
        check_o(o[b], w[0], b)
        if 0 <= c < 9:
            state[c] = S1.float()
    assert rel(x.now, state) <= FP32
    same = [0, 2, 3, 7, 8]
    assert torch.equal(x.now[same].cpu(), x.state[same])


def test_update_decays():
    """Growth, decays that vanish and -inf, which forgets the state."""
    print("update decays", flush=True)
    g = torch.tensor([0.0, 1.5, -80.0, -200.0, float("-inf"), -1e30])
    x = Setup(6, 2, 6, 3, 32, 32, 2, decay=lambda _: g.expand(2, 6).contiguous())
    o = S.damp_linear_update(x.pool, 0, i32([1, 0]), *x.dev, x.g.cuda())
    x.scale = 1.0
    for b, s in enumerate([1, 0]):
        w, S1 = x.want(b, 1, s)
        check_o(o[b], w[0])
        assert rel(x.now[s], S1) <= FP32


# ------------------------------------------------------------------ prompts

def run_prompts(x, lens, slot_in, slot_out, *, o_type=torch.float32, starts=None, max_len=None,
                workspace=None, poison=False, check=check_o):
    """Runs packed prompts and checks outputs (by `check`) and every state of
    the pool."""
    slots = x.state.shape[0]
    starts = np.concatenate([[0], np.cumsum(lens)[:-1]]) if starts is None else starts
    o = torch.full((x.n, x.HV, x.dv), 7.0, dtype=o_type, device="cuda")
    max_len = max(lens) if max_len is None else max_len
    S.damp_linear_prefill(x.pool, 0, i32(slot_in), *x.dev, x.g.cuda(), i32(starts), i32(lens),
                          max_len, slot_out=None if slot_out is None else i32(slot_out),
                          scale=x.scale, o=o, workspace=workspace)
    state, covered = x.state.clone(), torch.zeros(x.n, dtype=torch.bool)
    want = torch.full((x.n, x.HV, x.dv), 7.0, dtype=torch.float64)
    for b, (at, n) in enumerate(zip(starts, lens)):
        n = max(0, min(n, max_len, x.n - at))
        covered[at:at + n] = True
        if slot_in[b] < -1 or slot_in[b] >= slots:
            want[at:at + n] = 0.0
            continue
        want[at:at + n], S1 = x.want(at, n, slot_in[b])
        into = (slot_in if slot_out is None else slot_out)[b]
        if 0 <= into < slots:
            state[into] = S1.float()
    check(o[covered], want[covered], lens)
    assert bool((o[~covered.cuda()] == 7.0).all())
    assert rel(x.now, state) <= FP32, lens
    return o


@pytest.mark.parametrize("dk,dv", SIZES)
@pytest.mark.parametrize("o_type", [torch.float32, torch.bfloat16])
def test_prompt_sizes(dk, dv, o_type):
    print(f"prompt {dk}x{dv} {o_type}", flush=True)
    lens = [70, 1, 0, 33, 129]
    x = Setup(11, sum(lens), 4, 2, dk, dv, 6, fused=dk == 64, const=dk == 96)
    run_prompts(x, lens, [0, 4, 2, -1, 1], [0, 4, 2, 3, 5], o_type=o_type)


@pytest.mark.parametrize("dk,dv", [(256, 64), (160, 128), (136, 32), (256, 256), (248, 200)])
@pytest.mark.parametrize("o_type", [torch.float32, torch.bfloat16])
def test_prompt_wide_keys(dk, dv, o_type):
    """Keys of more than 128 channels, whose states take most of a wave's
    registers: one chunk and several, from zero states and old ones, whole and
    in segments."""
    print(f"prompt wide {dk}x{dv} {o_type}", flush=True)
    for seed, lens in enumerate([[20], [64], [65, 190], [700]]):
        B = len(lens)
        x = Setup(40 + seed, sum(lens), 2, 1, dk, dv, 2 * B)
        run_prompts(x, lens, [-1 if seed % 2 else 2 * b for b in range(B)],
                    [2 * b + 1 for b in range(B)], o_type=o_type)


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257,
                               1000])
def test_prompt_lengths(T):
    print(f"prompt length {T}", flush=True)
    for HV, HK, slot in ((2, 1, 1), (3, 3, -1)):
        x = Setup(T, T, HV, HK, 128, 128, 2)
        run_prompts(x, [T], [slot], [0])


@pytest.mark.parametrize("T,B,HV", [(5000, 1, 1), (3333, 2, 2), (9001, 1, 2)])
@pytest.mark.parametrize("o_type", [torch.float32, torch.bfloat16])
def test_prompt_long(T, B, HV, o_type):
    """Few long prompts, in place: the work is split along the tokens."""
    print(f"prompt long {T} {B} {HV}", flush=True)
    x = Setup(T, T * B, HV, 1, 64, 64, B)
    run_prompts(x, [T] * B, list(range(B)), None, o_type=o_type)


def test_prompt_ragged_beside_a_long_one():
    """A split made for the longest request, over requests that end in its
    first parts, at its edges and before it."""
    print("prompt ragged", flush=True)
    lens = [4100, 1, 0, 511, 512, 513, 1024, 2049]
    x = Setup(21, sum(lens), 2, 1, 64, 64, 9)
    run_prompts(x, lens, [0, 1, 2, 3, 4, 5, -1, 7], [0, 1, 8, 3, 4, 5, 6, 7])


def test_prompt_slots():
    """Padded requests (zeros), states not kept, one prefix continued by
    several requests, a copy by a request of length 0."""
    print("prompt slots", flush=True)
    lens = [40, 65, 30, 20, 0, 0, 90, 10]
    x = Setup(22, sum(lens), 4, 2, 64, 64, 8)
    run_prompts(x, lens, [3, 3, -5, 8, 3, -1, 0, -1], [4, 5, 6, 7, 1, 2, -1, 99])


def test_prompt_gaps_order_and_bounds():
    """Requests out of order with gaps between them that hold NaN, and starts
    and lengths beyond the token axis, which are cut."""
    print("prompt gaps", flush=True)
    x = Setup(23, 300, 2, 2, 64, 64, 8)
    starts, lens = [200, 10, 120, 290, 0], [50, 77, 1, 10, 5]
    covered = torch.zeros(300, dtype=torch.bool)
    for a, n in zip(starts, lens):
        covered[a:a + n] = True
    for t in x.dev:
        t[~covered.cuda()] = float("nan")
    x.g[~covered] = float("nan")
    run_prompts(x, lens, [0, 1, 2, 3, -1], [0, 1, 2, 3, 4], starts=starts)
    x = Setup(24, 100, 2, 2, 64, 64, 8)
    o = torch.full((100, 2, 64), 7.0, device="cuda")
    S.damp_linear_prefill(x.pool, 0, i32([0, 1, 2, 3, 4]), *x.dev, x.g.cuda(),
                          i32([95, -3, 101, 40, 0]), i32([50, 9, 9, -2, 1000]), 30, o=o,
                          scale=x.scale)
    state = x.state.clone()
    for b, at, n in ((0, 95, 5), (4, 0, 30)):
        w, S1 = x.want(at, n, b)
        check_o(o[at:at + n], w)
        state[b] = S1.float()
    assert bool((o[30:95] == 7.0).all())
    assert rel(x.now, state) <= FP32
    assert torch.equal(x.now[[1, 2, 3]].cpu(), x.state[[1, 2, 3]])


def test_prompt_decays():
    """Heads that never forget, that grow, that forget within a token, resets
    (-inf) inside and at the edges of a chunk, and steep decays beside them."""
    print("prompt decays", flush=True)
    T = 200

    def decay(g):
        g = g.clone()
        g[:, 0] = 0.0
        g[:, 1] = 0.01
        g[:, 2] = -30.0
        g[[0, 1, 63, 64, 100, 127, 199], 3] = float("-inf")
        g[::3, 4] = -500.0
        g[:, 5] = -1e30
        return g

    x = Setup(25, T, 6, 2, 64, 64, 2, decay=decay)
    run_prompts(x, [T], [1], [0])
    x = Setup(26, 2 * T, 6, 3, 128, 64, 2, decay=lambda g: torch.cat([decay(g[:T]), decay(g[T:])]))
    run_prompts(x, [T + 3, T - 3], [0, -1], [0, 1])


def check_terms(x, o, start, length, slot):
    """bf16 outputs of one request: half a step of bf16, and of the sum of the
    terms' absolute values 2^-17 and fp32's. (Two bf16 parts leave at most 2^-16
    of a term; not of every term, nor with one sign.)"""
    q, k, v = (t[start:start + length].abs() for t in x.cpu)
    S0 = x.state[slot].abs() if slot >= 0 else torch.zeros_like(x.state[0])
    terms, _ = ref.linear(q, k, v, x.g[start:start + length], S0, x.scale)
    want, _ = x.want(start, length, slot)
    got = o[start:start + length].double().cpu()
    assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -17 + FP32) * terms).all())


GROWTH = {  # log-decays [T] and whether values are 0 while they grow
    # a new request whose first values are 0: its state stays 0 whatever grows
    "zeros": (lambda t: torch.where(t < 150, 3.0, -0.1), True),
    # a state of 1e-30 that grows by e^100
    "tiny": (lambda t: torch.where(t < 150, 100 / 150, -0.1), True),
    # steady growth, e^60 in all
    "steady": (lambda t: torch.full(t.shape, 60 / len(t)), False),
    # single tokens that grow by more than a chunk may, and back
    "back and forth": (lambda t: torch.where(t % 2 == 0, 30.0, -30.0), False),
    # one large factor a token, each forgotten by the next
    "resets": (lambda t: torch.where(t % 3 == 1, 60.0, float("-inf")), False),
    # growth in one token of many
    "single": (lambda t: torch.where(t % 50 == 49, 20.0, -1.0), False),
}


@pytest.mark.parametrize("what", GROWTH)
@pytest.mark.parametrize("T,dk,dv,HV", [(200, 64, 64, 2), (40, 128, 128, 2), (200, 128, 128, 4),
                                        (700, 128, 48, 2), (300, 256, 72, 1)])
@pytest.mark.parametrize("o_type", [torch.float32, torch.bfloat16])
def test_prompt_growth(what, T, dk, dv, HV, o_type):
    """Positive log-decays: the factor of many tokens may leave fp32 where the
    recurrence, whose states are 0, tiny or forgotten, does not. bf16 outputs
    are bounded by the sizes of their own terms: rows differ by many orders
    here, and a state that one token dominates leaves rows in which all terms
    cancel."""
    print(f"prompt growth {what} {T} {dk}x{dv} {HV} {o_type}", flush=True)
    g, quiet = GROWTH[what]
    t = torch.arange(T)
    # the first head grows, the others decay beside it
    x = Setup(50, T, HV, 1, dk, dv, 2, decay=lambda d: torch.cat([g(t)[:, None], d[:, 1:]], 1))
    if quiet:
        x.cpu[2][:150, 0] = 0.0
        x.dev[2] = x.cpu[2].contiguous().cuda()
    if what == "tiny":
        x.state[:, 0] *= 1e-30
        x.now.copy_(x.state)
    slot = -1 if what == "zeros" else 1
    if o_type is torch.bfloat16:
        o = run_prompts(x, [T], [slot], [0], o_type=o_type, check=lambda *_: None)
        check_terms(x, o, 0, T, slot)
        return
    o = run_prompts(x, [T], [slot], [0])
    w, S1 = x.want(0, T, slot)
    for h in range(HV):  # each head on its own: growth makes them unlike
        assert rel(o[:, h], w[:, h]) <= FP32 and rel(x.now[0, h], S1[h]) <= FP32, h


def test_prompt_growth_beside_others():
    """Requests of one call whose chunks end at different tokens."""
    print("prompt growth beside", flush=True)
    lens = [200, 64, 130, 1, 500]
    n = sum(lens)

    def decay(g):
        g = g.clone()
        g[50:150, 1] = 0.5
        g[264:394:7, 0] = 25.0
        g[264 + 3:394:7, 0] = -25.0
        g[400:500] = 0.2
        return g

    x = Setup(51, n, 4, 2, 128, 128, 10, decay=decay)
    run_prompts(x, lens, [0, 1, 2, 3, 4], [5, 6, 2, 8, 9])
    x = Setup(51, n, 4, 2, 128, 128, 10, decay=decay)
    o = run_prompts(x, lens, [0, 1, 2, 3, 4], [5, 6, 2, 8, -1], o_type=torch.bfloat16,
                    check=lambda *_: None)
    for b, at in enumerate([0, 200, 264, 394, 395]):
        check_terms(x, o, at, lens[b], b)


def test_prompt_resets_keep_precision():
    """After many resets and steep decays the running sum of log-decays is in
    the thousands; what decays between two later tokens keeps fp32's digits."""
    print("prompt resets", flush=True)
    x = Setup(27, 256, 2, 2, 64, 64, 1,
              decay=lambda g: torch.where(torch.arange(256)[:, None] % 4 == 3, -150.0, g))
    run_prompts(x, [256], [0], None)


def test_prompt_values_of_any_size():
    """Large and tiny operands: nothing is scaled by an input's magnitude."""
    print("prompt magnitudes", flush=True)
    x = Setup(28, 150, 2, 1, 64, 64, 1)
    for i, f in ((0, 1e4), (1, 3e-6), (2, 1e9)):
        x.cpu[i] = (x.cpu[i].float() * f).bfloat16()
        x.dev[i] = x.cpu[i].contiguous().cuda()
    run_prompts(x, [150], [-1], [0])


def test_prompt_equals_its_parts():
    """A prompt in one call, in two calls, and token by token."""
    print("prompt parts", flush=True)
    x = Setup(29, 150, 4, 2, 128, 128, 3)
    g = x.g.cuda()
    x.now.zero_()
    whole = S.damp_linear_prefill(x.pool, 0, i32([0]), *x.dev, g, i32([0]), i32([150]), 150)
    a = S.damp_linear_prefill(x.pool, 0, i32([1]), *x.dev, g, i32([0]), i32([101]), 101)
    b = S.damp_linear_prefill(x.pool, 0, i32([1]), *x.dev, g, i32([101]), i32([49]), 49)
    assert rel(torch.cat([a[:101], b[101:]]), whole) <= 2 * FP32
    for t in range(150):
        o = S.damp_linear_update(x.pool, 0, i32([2]), *(y[t:t + 1] for y in x.dev), g[t:t + 1])
        assert rel(o[0], whole[t]) <= 20 * FP32
    assert rel(x.now[1], x.now[0]) <= 2 * FP32 and rel(x.now[2], x.now[0]) <= 2 * FP32


def test_offsets_beyond_32_bits():
    """Token rows, outputs and states whose byte offsets pass 2^32."""
    print("offsets", flush=True)
    n, stride = 70000, 32768
    wide = torch.empty(n, stride, dtype=torch.bfloat16, device="cuda")  # 4.6 GB
    x = Setup(31, 80, 2, 2, 64, 64, 4)
    at = n - 80
    rows = []
    for i, t in enumerate(x.dev):
        view = wide[:, 256 * i:256 * i + 128].unflatten(1, (2, 64))
        view[at:] = t
        rows.append(view)
    g = torch.zeros(n, 2, device="cuda")
    g[at:] = x.g.cuda()
    o = S.damp_linear_prefill(x.pool, 0, i32([2]), *rows, g, i32([at]), i32([80]), 80,
                              scale=x.scale)
    w, S1 = x.want(0, 80, 2)
    check_o(o[at:], w)
    assert rel(x.now[2], S1) <= FP32
    del wide, rows, o
    slots = 2200  # of 2 MiB
    buffer = torch.empty(slots * 32 * 128 * 128 * 4, dtype=torch.uint8, device="cuda")
    pool = D.Pool(D.damp_layout_init(128, 128, 0, D.DAMP_STATE_FP32), 1, slots, 32, buffer=buffer)
    now = buffer.view(torch.float32).view(slots, 32, 128, 128)
    x = Setup(32, 3, 32, 16, 128, 128, 3)
    src = [slots - 1, slots - 2, 5]
    now[src] = x.state.cuda()
    o = S.damp_linear_update(pool, 0, i32(src), *x.dev, x.g.cuda(), scale=x.scale)
    for b in range(3):
        w, S1 = x.want(b, 1, b)
        check_o(o[b], w[0])
        assert rel(now[src[b]], S1) <= FP32


def test_streams_and_graphs():
    """Calls on a side stream, and captured: every replay against eager."""
    print("graph", flush=True)
    lens = [200, 64, 0, 131]
    x = Setup(33, sum(lens), 4, 2, 64, 64, 8)
    g, starts = x.g.cuda(), i32(np.concatenate([[0], np.cumsum(lens)[:-1]]))
    ids, ls = i32([0, 1, 2, 3]), i32(lens)
    ws = torch.empty(S.damp_linear_prefill_workspace_bytes(x.pool, 4, 200), dtype=torch.uint8,
                     device="cuda")
    o, o1 = torch.empty(x.n, 4, 64, device="cuda"), torch.empty(4, 4, 64, device="cuda")

    def both():
        S.damp_linear_prefill(x.pool, 0, ids, *x.dev, g, starts, ls, 200, o=o, workspace=ws)
        S.damp_linear_update(x.pool, 0, ids, *(t[:4] for t in x.dev), g[:4], o=o1)

    first = x.now.clone()
    want = []
    for _ in range(4):
        both()
        torch.cuda.synchronize()
        want.append((o.clone(), o1.clone(), x.now.clone()))
    x.now.copy_(first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((o, o1, x.now), want[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    x.now.copy_(first)
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((o, o1, x.now), want[i])), i
        torch.randn(1000, device="cuda").sum().item()


def check_states(x, slot_in, slot_out, starts, lens):
    """Every written state by its own norm, every other one to the bit."""
    slots, written = x.state.shape[0], set()
    for b, (a, c) in enumerate(zip(slot_in, slot_out)):
        if -1 <= a < slots and 0 <= c < slots:
            _, S1 = x.want(starts[b], lens[b], a)
            written.add(c)
            for h in range(x.HV):
                assert rel(x.now[c, h], S1[h]) <= FP32, (b, h)
    rest = [s for s in range(slots) if s not in written]
    assert torch.equal(x.now[rest].cpu(), x.state[rest])


@pytest.mark.parametrize("HV,HK,dk,dv", [(32, 16, 128, 128), (32, 32, 128, 64), (16, 1, 256, 256),
                                         (24, 8, 64, 128)])
@pytest.mark.parametrize("o_type", [torch.float32, torch.bfloat16])
def test_prompt_heads_of_a_model(HV, HK, dk, dv, o_type):
    """As many heads as models have: several workgroups of a head, heads that
    share keys in the order of the XCDs, whole and cut into segments; the same
    bits on every run."""
    print(f"prompt heads {HV} {HK} {dk}x{dv} {o_type}", flush=True)
    for seed, lens in ((60, [300, 2, 65]), (61, [33] * 5)):
        B = len(lens)
        x = Setup(seed, sum(lens), HV, HK, dk, dv, 2 * B, fused=True)
        starts = np.concatenate([[0], np.cumsum(lens)[:-1]])
        slot_in, slot_out = list(range(B)), list(range(B, 2 * B))
        o = run_prompts(x, lens, slot_in, slot_out, o_type=o_type)
        check_states(x, slot_in, slot_out, starts, lens)
        state = x.now.clone()
        again = run_prompts(x, lens, slot_in, slot_out, o_type=o_type)
        assert torch.equal(o, again) and torch.equal(state, x.now)


@pytest.mark.parametrize("T,HV,dk,dv", [(1, 3, 128, 128), (1, 2, 64, 64), (63, 3, 128, 128),
                                        (65, 2, 256, 40), (200, 2, 16, 16)])
def test_prompt_states_by_slot(T, HV, dk, dv):
    """Small states in a pool of larger ones."""
    print(f"prompt states {T} {HV} {dk}x{dv}", flush=True)
    x = Setup(62 + T, 2 * T, HV, 1, dk, dv, 7)
    slot_in, slot_out = [-1, 4], [5, 4]
    run_prompts(x, [T, T], slot_in, slot_out)
    check_states(x, slot_in, slot_out, [0, T], [T, T])


@pytest.mark.parametrize("o_type", [torch.float32, torch.bfloat16])
def test_prompt_slots_in_segments(o_type):
    """Padded requests, states that are not kept, one state continued by several
    requests and a copy by a request of length 0, in a call whose requests are
    cut into segments."""
    print(f"prompt slots in segments {o_type}", flush=True)
    lens = [700, 300, 513, 400, 1, 600, 0, 129]
    starts = np.concatenate([[0], np.cumsum(lens)[:-1]])
    x = Setup(70, sum(lens), 2, 1, 64, 64, 12)
    assert S.damp_linear_prefill_workspace_bytes(x.pool, len(lens), max(lens)) > 0
    slot_in, slot_out = [3, 3, -5, 12, 3, -1, 3, 0], [4, -1, 6, 7, 8, -1, 9, 0]
    run_prompts(x, lens, slot_in, slot_out, o_type=o_type)
    check_states(x, slot_in, slot_out, starts, lens)


def test_decays_in_wider_rows():
    """g_stride above HV: decays left in a wider row of a projection."""
    print("g stride", flush=True)
    n, HV = 333, 3
    x = Setup(71, n, HV, 1, 64, 64, 4)
    wide = torch.full((n, 11), float("nan"), device="cuda")
    wide[:, 4:4 + HV] = x.g.cuda()
    g = wide[:, 4:]
    q, k, v = x.dev
    o, ws = torch.empty(n, HV, 64, device="cuda"), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    at = lambda t: t.data_ptr()  # noqa: E731
    ids, into, start, lens = i32([1]), i32([2]), i32([0]), i32([n])
    operands = [1, at(q), 64, at(k), 64, at(v), 64 * HV, at(g), 11, x.scale, at(o), D.DAMP_DT_FP32]
    stream = torch.cuda.current_stream().cuda_stream
    assert S.damp_linear_prefill_workspace_bytes(x.pool, 1, n) <= ws.numel()
    D._check(S.lib().damp_linear_prefill(ctypes.byref(x.pool.desc), 0, at(ids), at(into), 1, n, n,
                                         at(start), at(lens), *operands, at(ws), ws.numel(), stream))
    w, S1 = x.want(0, n, 1)
    check_o(o, w)
    assert rel(x.now[2], S1) <= FP32
    x.now.copy_(x.state)
    slots = i32([0, 1, 2])
    D._check(S.lib().damp_linear_update(ctypes.byref(x.pool.desc), 0, at(slots), None, 3, *operands,
                                        stream))
    for b in range(3):
        w, S1 = x.want(b, 1, b)
        check_o(o[b], w[0])
        assert rel(x.now[b], S1) <= FP32


def test_a_stream_of_the_callers_with_the_bindings_scratch():
    """Calls on a stream that is not torch's current one, outputs and scratch
    allocated by the binding, while the current stream takes and frees memory:
    the same results as on the current stream."""
    print("own stream", flush=True)
    lens = [700, 1, 64]
    x = Setup(36, sum(lens), 4, 2, 64, 64, 3)
    g, starts = x.g.cuda(), i32(np.concatenate([[0], np.cumsum(lens)[:-1]]))
    ids, ls = i32([0, 1, 2]), i32(lens)
    gen = torch.Generator(device="cuda").manual_seed(0)
    p = torch.softmax(torch.randn(8, 4, 9000, generator=gen, device="cuda"), -1)
    q = torch.softmax(torch.randn(8, 3, 9000, generator=gen, device="cuda"), -1)
    drafts = torch.randint(0, 9000, (8, 3), generator=gen, device="cuda", dtype=torch.int32)
    u = torch.rand(8, 4, generator=gen, device="cuda")
    refs, first = i32([0, 1, 2]), x.now.clone()

    def turn(stream=None):
        r, kw = refs.clone(), dict(stream=stream)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        o = S.damp_linear_prefill(x.pool, 0, ids, *x.dev, g, starts, ls, 700, **kw)
        o1 = S.damp_linear_update(x.pool, 0, ids, *(t[:3] for t in x.dev), g[:3], **kw)
        a, out = S.damp_verify_drafts(p, q, drafts, u, **kw)
        where, live = S.damp_slots_compact(x.pool, r, **kw)
        if stream is not None:
            for _ in range(8):  # what the calls above gave back is not the current stream's to take
                torch.full((1 << 20,), -1, dtype=torch.int32, device="cuda")
            stream.synchronize()
        torch.cuda.synchronize()
        return o, o1, a, out, where, live, r, x.now.clone()

    want = turn()
    assert S.damp_linear_prefill_workspace_bytes(x.pool, 3, 700) > 0
    side = torch.cuda.Stream()
    for i in range(3):
        x.now.copy_(first)
        got = turn(side)
        assert all(torch.equal(s, t) for s, t in zip(got, want)), i


def test_binding_refusals():
    x = Setup(34, 4, 4, 2, 64, 64, 4)
    g, ids = x.g.cuda(), i32([0, 1, 2, 3])
    q, k, v = x.dev
    with pytest.raises(ValueError, match="k has shape"):
        S.damp_linear_update(x.pool, 0, ids, q, k[:, :1], v, g)
    with pytest.raises(ValueError, match="heads of a token"):
        S.damp_linear_update(x.pool, 0, ids, q.transpose(1, 2).contiguous().transpose(1, 2), k, v, g)
    with pytest.raises(ValueError, match="bfloat16"):
        S.damp_linear_update(x.pool, 0, ids, q.float(), k, v, g)
    with pytest.raises(ValueError, match="g"):
        S.damp_linear_update(x.pool, 0, ids, q, k, v, g.bfloat16())
    with pytest.raises(ValueError, match="slot_in"):
        S.damp_linear_update(x.pool, 0, ids[:3], q, k, v, g)
    with pytest.raises(D.DampError, match="distances"):
        S.damp_linear_update(x.pool, 0, ids, q, k[:1].expand(4, 2, 64), v, g)
    mixed = D.Pool(D.damp_layout_init(64, 64, 8), 1, 4, 4)
    with pytest.raises(D.DampError, match="FP32 pool") as e:
        S.damp_linear_update(mixed, 0, ids, q, k, v, g)
    assert e.value.status == D.DAMP_ERR_UNSUPPORTED


def test_checked_slots(monkeypatch):
    """With DAMP_CHECK_SLOTS set a batch that races on a state is refused."""
    x = Setup(35, 3, 2, 2, 32, 32, 6)
    g = x.g.cuda()
    monkeypatch.setenv("DAMP_CHECK_SLOTS", "1")
    before = x.now.clone()
    for slot_in, slot_out, what in (([0, 1, 0], None, "more than once"),
                                    ([0, 1, 2], [3, 4, 3], "more than once"),
                                    ([0, 1, 2], [1, 3, 4], "written for entry 0 and read for 1")):
        with pytest.raises(D.DampError, match=what):
            S.damp_linear_update(x.pool, 0, i32(slot_in), *x.dev, g,
                                 slot_out=None if slot_out is None else i32(slot_out))
    assert torch.equal(x.now, before)
    S.damp_linear_update(x.pool, 0, i32([0, 0, 2]), *x.dev, g, slot_out=i32([3, 4, 2]))
