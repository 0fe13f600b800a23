"""Host-side checks of the serving operators: exports, workspace sizes and
refusals. No GPU needed: every call fails validation or has nothing to do."""
import contextlib
import ctypes
import glob
import os
import re
import shutil
import subprocess
import types

import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2608_27513_amd import damp as D
from paper_2608_27513_amd import serving as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "damp_serving.h")
P = ctypes.c_void_p(0x7f0000100000)  # never dereferenced
ODD = ctypes.c_void_p(0x7f0000100008)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(D.LIB_PATH):
        from paper_2608_27513_amd import build
        build.build()
    return S.lib()


def pool_of(dk=64, dv=64, kind=D.DAMP_STATE_FP32, layers=2, slots=4, hv=8):
    lay = D.damp_layout_init(dk, dv, 0, kind)
    pool = D.damp_pool()
    need = D.damp_pool_required_bytes(lay, layers, slots, hv)
    assert D.lib().damp_pool_init(ctypes.byref(pool), ctypes.byref(lay), layers, slots, hv,
                                  ctypes.c_void_p(0x7f0000000000), need) == 0
    return pool


def status(fn, *args):
    return fn(*args), D.lib().damp_last_error().decode()


def test_every_declared_symbol_is_exported(L):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(damp_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(S.EXPORTS)
    for n in names:
        assert hasattr(L, n), n


# the arguments num_k_heads .. o_dtype of both linear-attention calls
OPERANDS = [4, P, 256, P, 256, P, 512, P, 8, 1.0, P, D.DAMP_DT_FP32]
BAD_OPERANDS = {"num_k_heads 3": (0, 3), "num_k_heads 0": (0, 0), "q": (1, None), "q odd": (1, ODD),
                "q_stride short": (2, 248), "q_stride odd": (2, 260), "k": (3, None),
                "k odd": (3, ODD), "k_stride 0": (4, 0), "v": (5, None), "v odd": (5, ODD),
                "v_stride": (6, 504), "v_stride negative": (6, -512), "g": (7, None),
                "g_stride 4": (8, 4), "g_stride negative": (8, -8), "o": (10, None),
                "o odd": (10, ODD), "o_dtype": (11, D.DAMP_DT_FP16), "q far": (2, 2 ** 62)}


@pytest.mark.parametrize("what", BAD_OPERANDS)
def test_linear_operands(L, what):
    pool = pool_of()
    args = list(OPERANDS)
    i, args[i] = BAD_OPERANDS[what]
    for st, msg in (status(L.damp_linear_update, ctypes.byref(pool), 0, P, P, 3, *args, None),
                    status(L.damp_linear_prefill, ctypes.byref(pool), 0, P, P, 3, 100, 50, P, P,
                           *args, P, 1 << 40, None)):
        assert st == D.DAMP_ERR_INVALID_ARG and msg


def test_linear_refusals(L):
    pool = pool_of()
    up = [ctypes.byref(pool), 0, P, None, 3, *OPERANDS, None]
    for i, val in ((0, None), (1, 2), (1, -1), (2, None), (4, -1), (4, 65536)):
        a = list(up)
        a[i] = val
        assert L.damp_linear_update(*a) == D.DAMP_ERR_INVALID_ARG, (i, val)
    a = list(up)
    a[4] = 0
    assert L.damp_linear_update(*a) == D.DAMP_OK
    pre = [ctypes.byref(pool), 0, P, None, 3, 100, 50, P, P, *OPERANDS, P, 1 << 40, None]
    for i, val in ((0, None), (1, 2), (2, None), (4, -1), (5, -1), (5, 2 ** 31), (6, -1), (6, 101),
                   (7, None), (8, None)):
        a = list(pre)
        a[i] = val
        assert L.damp_linear_prefill(*a) == D.DAMP_ERR_INVALID_ARG, (i, val)
    a = list(pre)
    a[4] = 0
    assert L.damp_linear_prefill(*a) == D.DAMP_OK
    for i, val in ((11, 2 ** 24), (13, 2 ** 24), (15, 2 ** 24), (17, 2 ** 23)):
        a = list(pre)  # rows whose chunk does not fit 31 bits
        a[i] = val
        st, msg = status(L.damp_linear_prefill, *a)
        assert st == D.DAMP_ERR_INVALID_ARG and "too long" in msg, i
    for bad in (pool_of(kind=D.DAMP_STATE_MIXED), pool_of(dk=60), pool_of(dv=264), pool_of(dv=4)):
        st, msg = status(L.damp_linear_update, ctypes.byref(bad), *up[1:])
        assert st == D.DAMP_ERR_UNSUPPORTED and "multiples of 8" in msg
        st, _ = status(L.damp_linear_prefill, ctypes.byref(bad), *pre[1:])
        assert st == D.DAMP_ERR_UNSUPPORTED


def test_prefill_workspace_holds_what_a_call_may_cut(L):
    """The state of each piece of a request, with its decay: one long request
    is cut into as many pieces as fill the device and not more, and short or
    many requests need nothing."""
    pool = pool_of(dk=128, dv=128, layers=1, slots=2, hv=32)
    need = lambda B, n: L.damp_linear_prefill_workspace_bytes(ctypes.byref(pool), B, n)  # noqa: E731
    piece = 32 * (128 * 128 * 4 + 8)
    assert need(1, 32768) == 16 * piece  # 16 x 32 heads: two workgroups a CU
    assert need(1, 1 << 20) == 16 * piece
    assert need(1, 512) == 4 * piece and need(1, 257) == 3 * piece
    assert need(1, 256) == 0 and need(1, 0) == 0 and need(512, 4096) == 0
    # refused with a byte less, whatever the number of tokens
    for n_tokens in (1000, 5000):
        args = [ctypes.byref(pool), 0, P, None, 1, n_tokens, 1000, P, P, 4, P, 512, P, 512, P, 4096,
                P, 32, 1.0, P, D.DAMP_DT_FP32, P, need(1, 1000) - 1, None]
        st, msg = status(L.damp_linear_prefill, *args)
        assert st == D.DAMP_ERR_INVALID_ARG and "workspace" in msg


def test_verify_refusals(L):
    need = L.damp_verify_workspace_bytes(4, 1000)
    assert need > 0
    for B, V in ((0, 10), (-1, 10), (65536, 10), (4, 0), (4, 2 ** 22 + 1)):
        assert L.damp_verify_workspace_bytes(B, V) == 0
    args = [P, P, D.DAMP_DT_FP32, P, None, P, 4, 3, 1000, P, P, P, need, None]
    for i, val in ((0, None), (1, None), (2, D.DAMP_DT_FP16), (3, None), (5, None), (6, -1),
                   (6, 65536), (7, -1), (7, 1025), (8, 0), (8, 2 ** 22 + 1), (9, None), (10, None),
                   (11, None), (11, ODD), (12, need - 1)):
        a = list(args)
        a[i] = val
        st, msg = status(L.damp_verify_drafts, *a)
        assert st == D.DAMP_ERR_INVALID_ARG and msg, (i, val)
    a = list(args)
    a[6] = 0
    assert L.damp_verify_drafts(*a) == D.DAMP_OK


def test_slots_refusals(L):
    for fn in (L.damp_slots_alloc, L.damp_slots_retain, L.damp_slots_release):
        for args in ((P, 0, P, 3), (P, -1, P, 3), (None, 8, P, 3), (P, 8, None, 3), (P, 8, P, -1)):
            assert fn(*args, None) == D.DAMP_ERR_INVALID_ARG
        assert fn(P, 8, P, 0, None) == D.DAMP_OK
    pool = ctypes.byref(pool_of())
    fork = [pool, -1, P, P, 3, 2, None]
    for i, val in ((0, None), (1, -2), (1, 2), (2, None), (3, None), (4, -1), (5, -1), (4, 2 ** 30)):
        a = list(fork)
        a[i] = val
        a[5] = 4 if (i, val) == (4, 2 ** 30) else a[5]
        assert L.damp_slots_fork(*a) == D.DAMP_ERR_INVALID_ARG, (i, val)
    for i in (4, 5):
        a = list(fork)
        a[i] = 0
        assert L.damp_slots_fork(*a) == D.DAMP_OK
    need = L.damp_slots_compact_workspace_bytes(pool)
    assert need >= 2 * 4 * 4 and L.damp_slots_compact_workspace_bytes(None) == 0
    comp = [pool, P, P, P, P, need, None]
    for i, val in ((0, None), (1, None), (2, None), (3, None), (4, None), (4, ODD), (5, need - 1)):
        a = list(comp)
        a[i] = val
        assert L.damp_slots_compact(*a) == D.DAMP_ERR_INVALID_ARG, (i, val)


# ------------------------------------------------------------ the built code

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def chunk_loops(listing):
    """{kernel: instructions of its outermost loops with matrix products} of the
    prompt kernels in a disassembly."""
    loops, name, code = {}, None, []

    def close():
        if name is None or "prompt_chunks" not in name:
            return
        at = {addr: i for i, (addr, _) in enumerate(code)}
        base, spans = code[0][0], []
        for i, (_, text) in enumerate(code):
            to = re.search(r"^s_c?branch\S* .*<\S+?(?:\+0x([0-9a-f]+))?>$", text)
            if to and at[base + int(to.group(1) or "0", 16)] <= i:
                spans.append((at[base + int(to.group(1) or "0", 16)], i))
        spans = [(a, b) for a, b in spans if any("v_mfma" in t for _, t in code[a:b + 1])]
        loops[name] = [t for i, (_, t) in enumerate(code) if any(a <= i <= b for a, b in spans)]

    for line in listing.splitlines():
        head = re.match(r"[0-9a-f]+ <(\S+)>:$", line)
        if head:
            close()
            name, code = head.group(1), []
        elif name and "//" in line:
            text, addr = line.split("//", 1)
            where = addr.split(":", 1)
            target = re.search(r"<\S+>", where[1])
            code.append((int(where[0], 16), text.strip() + (" " + target.group(0) if target else "")))
    close()
    return loops


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_chunk_loops_have_no_branch_by_the_mask(L, tmp_path):
    """In a branch that only some lanes take, a register saved at its head's
    join is lost to the others: seen in a build of the prompt kernel whose
    registers were short. Its chunk loops hold none, in any of its forms."""
    lib = shutil.copy(D.LIB_PATH, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True)
    loops = {}
    for f in glob.glob(lib + ".*gfx950"):
        code = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", f], check=True,
                              capture_output=True, text=True).stdout
        loops.update(chunk_loops(code))
    assert len(loops) == 18  # d_k to 64, 128, 256; two and four waves; three sets of parts
    for name, code in loops.items():
        assert sum("v_mfma" in t for t in code) >= 24, name
        assert not [t for t in code if "saveexec" in t or "s_cbranch_execz" in t], name


def test_the_reader_of_loops_sees_a_branch_by_the_mask():
    listing = """
0000000000001000 <a_prompt_chunks_a>:
\ts_mov_b32 s0, 0   // 000000001000:
\tv_mfma_f32_32x32x16_bf16 v[0:15], v[0:3], v[4:7], v[0:15]   // 000000001004:
\ts_and_saveexec_b64 s[0:1], vcc   // 00000000100C:
\ts_cbranch_scc1 65532   // 000000001010: <a_prompt_chunks_a+0x4>
\ts_endpgm   // 000000001014:
"""
    loops = chunk_loops(listing)
    assert [t.split()[0] for t in loops["a_prompt_chunks_a"]] == [
        "v_mfma_f32_32x32x16_bf16", "s_and_saveexec_b64", "s_cbranch_scc1"]


# ------------------------------------------------ what the binding allocates

class FakeStream:
    cuda_stream = 0x1234


@pytest.mark.parametrize("stream", [None, FakeStream()])
def test_allocations_are_made_on_the_calls_stream(L, monkeypatch, stream):
    """Outputs and scratch that the binding allocates, and the zeros that the
    verification's has to start with, are made while the call's stream is
    torch's current one."""
    current, made, launched = [None], [], []

    @contextlib.contextmanager
    def on(s):
        before, current[0] = current[0], s
        yield
        current[0] = before

    def recorded(make):
        def run(shape, **kw):
            made.append(current[0])
            return make(shape, dtype=kw["dtype"])
        return run

    class Calls:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return lambda *a: 64
            return lambda *a: launched.append((name, a[-1])) or 0

    empty, zeros, i32 = torch.empty, torch.zeros, torch.int32
    layout = D.damp_layout_init(64, 64, 0, D.DAMP_STATE_FP32)
    pool = types.SimpleNamespace(num_v_heads=2, num_slots=4, layout=layout, desc=D.damp_pool())
    q = zeros(4, 2, 64, dtype=torch.bfloat16)
    g, ids, refs = zeros(4, 2), zeros(4, dtype=i32), zeros(4, dtype=i32)
    p, u = zeros(4, 2, 8), zeros(4, 2)
    drafts, names = zeros(4, 1, 8), zeros(4, 1, dtype=i32)
    monkeypatch.setattr(S, "lib", Calls)
    monkeypatch.setattr(S, "_at", lambda t, *a: t.data_ptr())
    monkeypatch.setattr(S, "_tokens", lambda t, name, n, h, d: (t.data_ptr(), h * d))
    monkeypatch.setattr(S, "_raw_stream", lambda s=None: 0 if s is None else s.cuda_stream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", recorded(empty))
    monkeypatch.setattr(torch, "zeros", recorded(zeros))
    for call, allocations in (
            (lambda **kw: S.damp_linear_update(pool, 0, ids, q, q, q, g, **kw), 1),
            (lambda **kw: S.damp_linear_prefill(pool, 0, ids, q, q, q, g, ids, ids, 1, **kw), 2),
            (lambda **kw: S.damp_verify_drafts(p, drafts, names, u, **kw), 3),
            (lambda **kw: S.damp_slots_alloc(refs, 3, **kw), 1),
            (lambda **kw: S.damp_slots_compact(pool, refs, **kw), 3)):
        made.clear()
        launched.clear()
        call(stream=stream)
        assert made == [stream] * allocations
        assert [s for _, s in launched] == [0 if stream is None else stream.cuda_stream]


# ----------------------------------------- the plain implementations themselves

def test_reference_recurrence_against_the_sum_over_tokens():
    """o_t = scale sum_j exp(g_{j+1} + .. + g_t) (q_t . k_j) v_j, from a zero state."""
    gen = torch.Generator().manual_seed(0)
    T, HV, HK, dk, dv = 9, 4, 2, 5, 3
    q, k = (torch.randn(T, HK, dk, generator=gen) for _ in range(2))
    v, g = torch.randn(T, HV, dv, generator=gen), -torch.rand(T, HV, generator=gen)
    o, _ = ref.linear(q, k, v, g, torch.zeros(HV, dk, dv), 0.5)
    for t in range(T):
        for h in range(HV):
            want = sum(float(torch.exp(g[j + 1:t + 1, h].double().sum()))
                       * float(q[t, h // 2].double() @ k[j, h // 2].double()) * v[j, h].double()
                       for j in range(t + 1)) * 0.5
            assert torch.allclose(o[t, h], want, rtol=1e-12)


def test_reference_verification_distributes_as_the_target():
    """Over many uniform numbers the first token follows p whatever q is."""
    rng = np.random.RandomState(1)
    V, n = 6, 40000
    p0 = np.array([0.3, 0.05, 0.25, 0.1, 0.2, 0.1])
    q0 = np.array([0.1, 0.3, 0.1, 0.1, 0.3, 0.1])
    p = np.broadcast_to(np.stack([p0, p0]), (n, 2, V))
    q = np.broadcast_to(q0, (n, 1, V))
    tokens = rng.choice(V, size=(n, 1), p=q0)
    u = rng.randint(0, 1 << 24, (n, 2)) / 2.0 ** 24
    a, out = ref.verify(p, q, tokens, u, np.ones(n, int))
    kept = a == 1
    assert np.abs(np.bincount(out[:, 0], minlength=V) / n - p0).max() <= 5 / np.sqrt(n)
    assert np.abs(np.bincount(out[kept, 1], minlength=V) / kept.sum() - p0).max() <= 5 / np.sqrt(n)
    assert abs(kept.mean() - np.minimum(p0, q0).sum()) <= 5 / np.sqrt(n)


def test_reference_compaction_keeps_every_live_slot():
    rng = np.random.RandomState(2)
    for _ in range(50):
        refs = rng.randint(0, 3, rng.randint(1, 30))
        where, new, live, moves = ref.compact(refs)
        assert sorted(where[where >= 0]) == list(range(live))
        assert (new[live:] == 0).all() and (new[:live] > 0).all()
        assert len(moves) == int((refs[:live] == 0).sum())
        for s in range(len(refs)):
            assert refs[s] == 0 or new[where[s]] == refs[s]
