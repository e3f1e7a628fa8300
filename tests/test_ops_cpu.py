"""Layers of another product than a matrix's (the gated product, the scaled
token embedding): the oracle against Eq. (1) and the sum-check's definition in
pure Python, the library's verifier on the oracle's proofs and on tampered
ones, and the calls' refusals that need no GPU."""
import copy
import ctypes
import gc
import weakref

import numpy as np
import pytest
import torch

from helpers import pack_planes
from oracle import oracle as orc
from paper_2505_17623_amd import inputs

P61 = (1 << 61) - 1


@pytest.fixture(scope="module")
def ra():
    from paper_2505_17623_amd import ra as ra_mod
    ra_mod.lib()
    return ra_mod


def eq(z, y):
    """eq(z, y) = prod z_i y_i + (1 - z_i)(1 - y_i) over field points (Eq. (1))."""
    out = 1
    for a, b in zip(z, y):
        out = out * (a * b + (1 - a) * (1 - b)) % P61
    return out


def bits_of(i, v):
    return [(i >> (v - 1 - j)) & 1 for j in range(v)]


def mle(table, z):
    v = len(z)
    return sum(int(t) * eq(z, bits_of(i, v)) for i, t in enumerate(table)) % P61


def round_values(f, v, deg, rho):
    """g_j(X) = sum over the remaining variables of f(rho_<j, X, y), from the definition."""
    out = []
    for j in range(v):
        for X in range(deg + 1):
            out.append(sum(f(rho[:j] + [X] + bits_of(y, v - 1 - j)) for y in range(1 << (v - 1 - j))) % P61)
    return out


@pytest.mark.parametrize("n,k", [(1, 1), (1, 4), (4, 1), (2, 4)])
def test_gate_oracle_is_the_definition(n, k):
    rng = np.random.default_rng(n * 10 + k)
    A, B = rng.integers(-2 ** 20, 2 ** 20, (2, n, k))
    chal = inputs.xorshift64_stream(11 + n, 200)
    o = orc.prove_gate_layer(A, B, 8, False, 0, chal, 3)
    v = (n * k).bit_length() - 1
    c = [int(x) for x in chal[3:3 + 2 * v]]
    r, rho = c[:v], c[v:]
    a, b = A.reshape(-1), B.reshape(-1)
    assert np.array_equal(o["C"], A * B)
    assert o["c0"] == mle(a * b, r)
    assert o["gate_evals"] == round_values(lambda z: eq(r, z) * mle(a, z) * mle(b, z), v, 3, rho)
    assert (o["a_at"], o["b_at"]) == (mle(a, rho), mle(b, rho))


@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (4, 3, 2), (2, 5, 3), (1, 8, 4)])
def test_embed_oracle_is_the_definition(n, vocab, d):
    rng = np.random.default_rng(vocab)
    tok = rng.integers(-1, vocab, n)
    E = rng.integers(-2 ** 15, 2 ** 15, (vocab, d))
    scale = -37
    chal = inputs.xorshift64_stream(5 + n, 200)
    o = orc.prove_embed_layer(tok, E, scale, 6, False, 1, chal, 2)
    ln, lk, lv = (n - 1).bit_length(), (d - 1).bit_length(), (vocab - 1).bit_length()
    c = [int(x) for x in chal[2:2 + ln + lk + lv]]
    r1, r2, rho = c[:ln], c[ln:ln + lk], c[ln + lk:]
    C = np.zeros((n, 1 << lk), dtype=np.int64)
    for i, t in enumerate(tok):
        if t >= 0:
            C[i, :d] = scale * E[t]
    assert np.array_equal(o["C"], C)
    W, e = [0] * (1 << lv), [0] * (1 << lv)
    for i, t in enumerate(tok):
        if t >= 0:
            W[t] = (W[t] + scale * eq(r1, bits_of(i, ln))) % P61
    for v in range(vocab):
        e[v] = sum(int(E[v, j]) * eq(r2, bits_of(j, lk)) for j in range(d)) % P61
    assert o["c0"] == mle(C.reshape(-1), r1 + r2) == sum(x * y for x, y in zip(W, e)) % P61
    assert o["mm_evals"] == round_values(lambda z: mle(W, z) * mle(e, z), lv, 2, rho)
    assert (o["a_star"], o["b_star"]) == (mle(W, rho), mle(e, rho))


def abi(res, **more):
    return dict(Z=res["Z"].astype(np.int32), R=res["R"].astype(np.int32), Rm=res["Rm"].astype(np.uint16),
                Y=res["Y"].astype(np.int32), bits=pack_planes(res["bits"]), transcript=res, **more)


def network(seed=91, n=4, vocab=11, d=6, hidden=8, s=8):
    """Tokens -> embedding -> gated block -> logits, proven by the oracle; the
    layers as ra_verify takes them."""
    rng = np.random.default_rng(seed)
    chal = inputs.xorshift64_stream(seed, 4000)
    k = 1 << (d - 1).bit_length()
    tok = rng.integers(0, vocab, n)
    tok[n - 1] = -1
    E = rng.integers(-600, 600, (vocab, d)).astype(np.int16)
    Wg, Wu = rng.integers(-300, 300, (2, k, hidden)).astype(np.int16)
    Wd, Wo = rng.integers(-300, 300, (hidden, k)).astype(np.int16), rng.integers(-300, 300, (k, 16)).astype(np.int16)
    e = orc.prove_embed_layer(tok, E, 700, s, False, 0, chal, 0)
    g = orc.prove_layer(e["Z"], Wg, s, True, 0, chal, e["cursor"])
    u = orc.prove_layer(e["Z"], Wu, s, False, 0, chal, g["cursor"])
    m = orc.prove_gate_layer(g["Z"], u["Z"], s, False, 0, chal, u["cursor"])
    w = orc.prove_layer(m["Z"], Wd, s, False, 0, chal, m["cursor"])
    o = orc.prove_layer(w["Z"], Wo, s, False, 0, chal, w["cursor"])
    i32 = lambda r: r["Z"].astype(np.int32)  # noqa: E731
    return seed, [abi(e, tokens=tok, B=E, scale=700), abi(g, A=i32(e), B=Wg, from_a=0), abi(u, A=i32(e), B=Wu, from_a=0),
                  abi(m, A=i32(g), B=i32(u), from_a=1, from_b=2), abi(w, A=i32(m), B=Wd, from_a=3),
                  abi(o, A=i32(w), B=Wo, from_a=4)]


def test_verifier_accepts_the_network(ra):
    seed, layers = network()
    assert ra.ra_verify(seed, layers) == (0, 0)
    assert ra.ra_verify(seed + 1, layers)[0] != 0


def test_verifier_accepts_single_entries(ra):
    chal = inputs.xorshift64_stream(3, 400)
    g = orc.prove_gate_layer([[5]], [[-7]], 1, True, 1, chal, 0)
    e = orc.prove_embed_layer([0], [[9]], 3, 1, False, 0, chal, g["cursor"])
    layers = [abi(g, A=np.array([[5]], dtype=np.int16), B=np.array([[-7]], dtype=np.int32)),
              abi(e, tokens=[0], B=np.array([[9]]), scale=3)]
    assert ra.ra_verify(3, layers) == (0, 0)


def change(layers, l, f):
    out = [dict(L, transcript=copy.copy(L["transcript"])) for L in layers]
    for key, v in out[l].items():
        if isinstance(v, np.ndarray):
            out[l][key] = v.copy()
    f(out[l])
    return out


def bump(key, i=None):
    def f(L):
        tr = L["transcript"]
        if i is None:
            tr[key] = (tr[key] + 1) % P61
        else:
            tr[key] = [(x + (q == i)) % P61 for q, x in enumerate(tr[key])]
    return f


def test_verifier_rejects_tampering(ra):
    seed, layers = network()

    def at(key, index, value):
        def f(L):
            L[key][index] = value
        return f
    E, G = 0, 3
    cases = [(E, bump("mm_evals", 0), 1), (E, bump("mm_evals", 7), 1), (E, bump("a_star"), 2), (E, bump("c0"), 1),
             (G, bump("gate_evals", 2), 1), (G, bump("gate_evals", 17), 1), (G, bump("a_at"), 2), (G, bump("c0"), 1),
             (E, at("B", (int(layers[0]["tokens"][0]), 0), 599), 3),
             (E, at("tokens", 0, (int(layers[0]["tokens"][0]) + 1) % 11), 3),
             (E, at("tokens", 1, -1), 3), (E, at("tokens", 0, 11), 13), (E, at("tokens", 0, -2), 13),
             (E, lambda L: L.update(scale=701), 3), (E, lambda L: L.update(from_a=0), 13),
             (G, at("A", (0, 1), 12345), 14), (G, at("B", (1, 1), 12345), 14),
             (G, lambda L: L.update(from_a=3), 14), (G, lambda L: L.update(from_a=2, from_b=1), 14),
             (G, lambda L: L.update(from_a=-2), 13),
             (1, lambda L: L.update(from_a=5), 14)]
    for l, f, want in cases:
        got = ra.ra_verify(seed, change(layers, l, f))
        assert got == (want, l), (l, want, got)
    # both final values changed so that their product holds: the openings catch it
    tr = layers[G]["transcript"]
    half = pow(2, P61 - 2, P61)
    bad = change(layers, G, lambda L: L["transcript"].update(a_at=tr["a_at"] * 2 % P61, b_at=tr["b_at"] * half % P61))
    assert ra.ra_verify(seed, bad) == (3, G)
    # a witness table changed behind a gated product
    assert ra.ra_verify(seed, change(layers, G, at("R", (0, 0), int(layers[G]["R"][0, 0]) + 1)))[1] == G


def test_gate_entries_beyond_the_field(ra):
    """(2^31 - 1)^2 exceeds 2^60: the product mod p no longer is the integer's."""
    seed, layers = network()

    def f(L):
        L["A"][0, 0] = L["B"][0, 0] = 2 ** 31 - 1
        L.update(from_a=-1, from_b=-1)
    assert ra.ra_verify(seed, change(layers, 3, f)) == (12, 3)


def test_workspace_sizes_and_null_arguments(ra):
    L, size = ra.lib(), ctypes.c_size_t()
    assert L.ra_gate_workspace_size(4, 8, None) == -1
    assert L.ra_gate_workspace_size(3, 8, ctypes.byref(size)) == -1
    assert L.ra_gate_workspace_size(1 << 16, 1 << 16, ctypes.byref(size)) == -9
    assert L.ra_embed_workspace_size(4, 0, 8, ctypes.byref(size)) == -1
    assert L.ra_embed_workspace_size(4, 8, 0, ctypes.byref(size)) == -1
    assert L.ra_embed_workspace_size(6, 8, 8, ctypes.byref(size)) == -1
    assert L.ra_embed_workspace_size(4, (1 << 22) + 1, 8, ctypes.byref(size)) == -9
    assert L.ra_embed_workspace_size(4, 8, (1 << 20) + 1, ctypes.byref(size)) == -9
    assert ra.gate_workspace_size(4, 8) > 0 and ra.embed_workspace_size(1, 7, 5) > 0
    assert ra.gate_workspace_size(1024, 4096) >= 2 * 8 * 1024 * 4096 // 2
    pr, mm = ra.GateProof(), ra.MatmulProof()
    assert L.ra_gate_prove(None, None, 1, 4, None, 1, 4, 4, 4, None, None, 0, ctypes.byref(pr)) == -1
    assert L.ra_embed_prove(None, None, 4, None, 4, 4, 4, 1, None, None, 0, ctypes.byref(mm)) == -1
    v, f = ctypes.c_int32(), ctypes.c_uint32()
    assert L.ra_verify_ops(P61, 1, 1, None, None, None, None, ctypes.byref(v), ctypes.byref(f)) == -1
    assert L.ra_verify_ops(P61, 0, 0, None, None, None, None, ctypes.byref(v), ctypes.byref(f)) == -5
    assert L.ra_verify_ops(97, 1, 0, None, None, None, None, ctypes.byref(v), ctypes.byref(f)) == -2


class Calls:
    """Stands in for the library: every entry point is logged and succeeds.
    `announced` says whether a witness announcement is open, as ra.h has it."""

    def __init__(self):
        self.log, self.announced = [], False

    def __getattr__(self, name):
        def call(h, *args):
            self.log.append(name)
            if name == "ra_witness_plan":
                self.announced = args[4] is not None
            return 0
        return call


@pytest.mark.parametrize("call", ["tokens", "shape", "type", "matrix", "raw matrix", "raw gate", "raw embed"])
def test_a_call_refused_in_python_leaves_no_witness_announced(ra, monkeypatch, call):
    """The layer's outputs may be freed after the refusal, so nothing may be
    left that would have a later layer's product write to them."""
    calls = Calls()
    monkeypatch.setattr(ra, "lib", lambda: calls)
    monkeypatch.setattr(ra, "_dptr", lambda t: ctypes.c_void_p(t.data_ptr()))
    ctx = ra.Context.__new__(ra.Context)
    ctx.h, ctx.deferred, ctx._fills, ctx._held = None, False, [], []
    I = torch.zeros((4, 8), dtype=torch.int32)  # noqa: E741
    S, tok = torch.zeros((4, 8), dtype=torch.int16), torch.zeros(4, dtype=torch.int64)
    bufs = {}
    refused = {"tokens": lambda: ra.prove_embed(ctx, tok, S, 3, 4, t=5, bufs=bufs),
               "shape": lambda: ra.prove_gate(ctx, I, I[:2], 4, t=5, bufs=bufs),
               "type": lambda: ra.prove_gate(ctx, I.double(), I, 4, t=5, bufs=bufs),
               "matrix": lambda: ra.prove_layer(ctx, I, I.T.contiguous(), 4, True, t=5, bufs=bufs),
               "raw matrix": lambda: ra.ra_sumcheck_matmul_prove(ctx, I, I.T.contiguous()),
               "raw gate": lambda: ra.ra_gate_prove(ctx, I, I, C=I),
               "raw embed": lambda: ra.ra_embed_prove(ctx, tok, S, 3)}[call]
    if call.startswith("raw"):
        ra.ra_witness_plan(ctx, 4, True, 0, 5, ra.witness_outputs(4, 4, "cpu"))
        assert calls.announced
    with pytest.raises((AssertionError, KeyError)):
        refused()
    assert "ra_witness_plan" in calls.log and not calls.announced, calls.log
    assert not any(name.endswith("_prove") for name in calls.log)


def test_an_announcement_is_withdrawn_by_null_buffers_only(ra):
    L = ra.lib()
    assert L.ra_witness_plan(None, 0, 0, 0, -1, None, None, None, None, None, 0) == -1


def gated_layer(A, B, seed=17):
    """One gated layer, proven by the oracle, as ra_verify takes it."""
    A, B = np.broadcast_arrays(np.asarray(A, dtype=np.int64), np.asarray(B, dtype=np.int64))
    return seed, abi(orc.prove_gate_layer(A.copy(), B.copy(), 8, False, 0, inputs.xorshift64_stream(seed, 400), 0))


@pytest.mark.parametrize("side", ["A", "B"])
def test_verifier_takes_one_row_of_a_gated_product_for_all(ra, side):
    """The prover's factors may be one row for all n (a learned scale); given to
    the verifier alone, it stands for n rows and is not read past its end."""
    rng = np.random.default_rng(2)
    full, row = rng.integers(-900, 900, (8, 4)).astype(np.int32), rng.integers(-900, 900, (1, 4)).astype(np.int16)
    seed, layer = gated_layer(*((row, full) if side == "A" else (full, row)))
    other = "B" if side == "A" else "A"
    assert ra.ra_verify(seed, [dict(layer, **{side: row, other: full})]) == (0, 0)
    bad = row.copy()
    bad[0, 3] += 1
    assert ra.ra_verify(seed, [dict(layer, **{side: bad, other: full})]) == (3, 0)


@pytest.mark.parametrize("dtype", [np.int8, np.uint16, np.int16, np.int32, np.int64, np.uint64])
def test_verifier_takes_a_gated_products_factors_in_any_integer_type(ra, dtype):
    rng = np.random.default_rng(4)
    A, B = rng.integers(0, 100, (2, 4, 8))
    seed, layer = gated_layer(A, B)
    for x, y in ((A.astype(dtype), B.astype(np.int32)), (A.astype(np.int32), B.astype(dtype)), (A.astype(dtype), B.astype(dtype))):
        assert ra.ra_verify(seed, [dict(layer, A=x, B=y)]) == (0, 0)


def test_verifier_refuses_other_factors_of_a_gated_product(ra):
    rng = np.random.default_rng(6)
    A, B = rng.integers(-100, 100, (2, 4, 8)).astype(np.int32)
    seed, layer = gated_layer(A, B)
    past = A.astype(np.int64)
    past[1, 2] = 2 ** 31
    for x, y in ((A[:, :4], B), (A, B[:, :4]), (A[:2], B), (A, B[:3]), (A.reshape(-1), B), (A, B[None]), (A, past), (past, B),
                 (A.astype(np.float16), B), (A, B.astype(np.float64)), (A, B.astype(bool))):
        with pytest.raises(ValueError):
            ra.ra_verify(seed, [dict(layer, A=x, B=y)])


def refused(ra, seed, layers):
    with pytest.raises(ValueError):
        ra.ra_verify(seed, layers)


@pytest.mark.parametrize("key,dtype", [("tokens", np.int32), ("B", np.int16), ("Z", np.int32), ("R", np.int32),
                                       ("Y", np.int32), ("Rm", np.uint16), ("bits", np.uint64)])
def test_verifier_reads_an_embeddings_arrays_as_they_are(ra, key, dtype):
    """A value that another type would not hold is not taken for the one it
    wraps to, an array of another size is not read past its end, and other
    integer types give the same verdict."""
    seed, layers = network()
    E, rest = layers[0], layers[1:]
    whole = np.asarray(E[key])
    wide = whole.astype(object) if key == "bits" else whole.astype(np.int64)
    if key != "bits":  # a uint64 holds every word
        assert ra.ra_verify(seed, [dict(E, **{key: wide}), *rest]) == (0, 0)
        wide = wide.copy()
        wide.flat[0] += 2 ** (8 * np.dtype(dtype).itemsize)
        refused(ra, seed, [dict(E, **{key: wide}), *rest])
    refused(ra, seed, [dict(E, **{key: whole.astype(np.float64)}), *rest])
    for part in (whole[:-1], np.concatenate([whole, whole])):
        if key == "B":  # another vocabulary is another statement, not a malformed one
            assert ra.ra_verify(seed, [dict(E, B=part), *rest])[0] != 0
        else:
            refused(ra, seed, [dict(E, **{key: part}), *rest])
    if key == "B":
        refused(ra, seed, [dict(E, B=whole.reshape(-1)), *rest])


def test_verifier_reads_a_matrix_layers_arrays_as_they_are(ra):
    rng = np.random.default_rng(8)
    A, B = rng.integers(-300, 300, (4, 8)), rng.integers(-300, 300, (8, 16))
    layer = abi(orc.prove_layer(A, B, 8, True, 0, inputs.xorshift64_stream(23, 400), 0), A=A, B=B)
    assert ra.ra_verify(23, [layer]) == (0, 0)  # int64 throughout
    past = [B.copy(), A.copy()]
    past[0][0, 0] += 1 << 16
    past[1][0, 0] += 1 << 32
    for bad in (dict(B=past[0]), dict(A=past[1]), dict(A=A[:, :4]), dict(B=B[:4]), dict(A=A.astype(np.float32)), dict(A=A[0]),
                dict(Z=layer["Z"][:2]), dict(Rm=layer["Rm"].astype(np.int64) - 1 - layer["Rm"].max()), dict(bits=layer["bits"][:-1])):
        refused(ra, 23, [dict(layer, **bad)])
    signed = dict(layer, Rm=layer["Rm"].view(np.int16), bits=layer["bits"].view(np.int64))
    assert ra.ra_verify(23, [signed]) == (0, 0)
    src = np.arange(32, dtype=np.int32)
    refused(ra, 23, [dict(layer, link_src=src[:-1])])


def test_verifier_over_fp2_reads_a_layers_arrays_as_they_are(ra):
    rng = np.random.default_rng(9)
    A, B = rng.integers(-300, 300, (2, 4)), rng.integers(-300, 300, (4, 2))
    chal = [(int(x), int(y)) for x, y in inputs.xorshift64_stream(29, 800).reshape(-1, 2)]
    layer = abi(orc.prove_layer_fp2(A, B, 8, True, 0, chal, 0), A=A, B=B)
    assert ra.ra_verify_fp2(29, [layer]) == (0, 0)
    for bad in (dict(A=A[:, :2]), dict(B=B + (1 << 16)), dict(A=A.astype(np.float32)), dict(Y=layer["Y"][:1])):
        with pytest.raises(ValueError):
            ra.ra_verify_fp2(29, [dict(layer, **bad)])


@pytest.mark.parametrize("scale", [700 + 2 ** 32, 2 ** 31, -(2 ** 31) - 1])
def test_a_scale_past_int32_is_refused(ra, monkeypatch, scale):
    """Not taken for the int32 it wraps to, by the verifier or by the prover."""
    seed, layers = network()
    assert layers[0]["scale"] == 700
    refused(ra, seed, [dict(layers[0], scale=scale), *layers[1:]])
    monkeypatch.setattr(ra, "_dptr", lambda t: ctypes.c_void_p(t.data_ptr()))
    calls = Calls()
    monkeypatch.setattr(ra, "lib", lambda: calls)
    ctx = ra.Context.__new__(ra.Context)
    ctx.h, ctx.deferred, ctx._fills, ctx._held = None, False, [], []
    tok, E = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 8), dtype=torch.int16)
    for call in (lambda: ra.prove_embed(ctx, tok, E, scale, 4, t=5), lambda: ra.ra_embed_prove(ctx, tok, E, scale)):
        with pytest.raises(ValueError):
            call()
    assert not any(name.endswith("_prove") for name in calls.log) and not calls.announced


def test_a_scale_that_is_no_integer_is_refused(ra):
    seed, layers = network()
    for scale in (700.0, 700.5, "700"):
        with pytest.raises(TypeError):
            ra.ra_verify(seed, [dict(layers[0], scale=scale), *layers[1:]])
    assert ra.ra_verify(seed, [dict(layers[0], scale=np.int64(700)), *layers[1:]]) == (0, 0)


@pytest.mark.parametrize("which", range(6))
def test_a_callers_outputs_of_another_size_or_type_are_refused(ra, monkeypatch, which):
    """Before anything is announced or called: the product's kernels write them."""
    calls = Calls()
    monkeypatch.setattr(ra, "lib", lambda: calls)
    monkeypatch.setattr(ra, "_dptr", lambda t: ctypes.c_void_p(t.data_ptr()))
    monkeypatch.setattr(ra, "_rows", lambda t: (ctypes.c_void_p(t.data_ptr()), t.stride(0)))
    ctx = ra.Context.__new__(ra.Context)
    ctx.h, ctx.deferred, ctx._fills, ctx._held = None, False, [], []
    tok, E = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 8), dtype=torch.int16)
    I = torch.zeros((4, 8), dtype=torch.int32)  # noqa: E741
    for change in (lambda x: x[:1], lambda x: x.to(torch.int8)):
        outs = [torch.empty((4, 8), dtype=torch.int64), *ra.witness_outputs(4, 8, "cpu")]
        outs[which] = change(outs[which])
        entries = [lambda b: ra.prove_embed(ctx, tok, E, 3, 4, t=5, bufs=b), lambda b: ra.prove_gate(ctx, I, I, 4, t=5, bufs=b),
                   lambda b: ra.prove_gate(ctx, I, I, 4, bufs=b), lambda b: ra.prove_layer(ctx, I[:, :4], E, 4, True, t=5, bufs=b)]
        if which > 0:  # an announcement has no C
            entries.append(lambda b: ra.ra_witness_plan(ctx, 4, True, 0, 5, b["wit"]))
        for call in entries:
            with pytest.raises(AssertionError):
                call({"C": outs[0], "wit": tuple(outs[1:])})
    assert not calls.announced and not any(name.endswith("_prove") for name in calls.log)


@pytest.mark.parametrize("kind", ["gate", "embed", "matrix"])
@pytest.mark.parametrize("refusing", ["ra_rescale_relu_witness", "ra_range_prove"])
def test_a_layer_refused_midway_keeps_what_the_library_still_fills(ra, monkeypatch, kind, refusing):
    """Deferred: the product's and the witness's structs and arrays are written
    at the next sync, so they stay although the layer's later call is refused."""
    structs = {}

    class Refusing(Calls):
        def __getattr__(self, name):
            def call(h, *args):
                if name == refusing:
                    return -9
                if name == "ra_rescale_relu_witness":
                    args[-1]._obj.P = 16  # known at once
                if args and hasattr(args[-1], "_obj"):
                    structs[name] = weakref.ref(args[-1]._obj)
                return 0
            return call
    calls = Refusing()
    monkeypatch.setattr(ra, "lib", lambda: calls)
    monkeypatch.setattr(ra, "_dptr", lambda t: ctypes.c_void_p(t.data_ptr()))
    monkeypatch.setattr(ra, "_rows", lambda t: (ctypes.c_void_p(t.data_ptr()), t.stride(0)))
    ctx = ra.Context.__new__(ra.Context)
    ctx.h, ctx.deferred, ctx._fills, ctx._held = None, True, [], []
    tok, E = torch.zeros(4, dtype=torch.int32), torch.zeros((4, 8), dtype=torch.int16)
    I = torch.zeros((4, 8), dtype=torch.int32)  # noqa: E741
    with pytest.raises(ra.RAError):
        if kind == "gate":
            ra.prove_gate(ctx, I, I, 8, t=3, plan=False)
        elif kind == "embed":
            ra.prove_embed(ctx, tok, E, 3, 8, t=3, plan=False)
        else:
            ra.prove_layer(ctx, I[:, :4], E, 8, False, t=3, plan=False)
    gc.collect()
    want = 1 if refusing == "ra_rescale_relu_witness" else 2
    assert len(structs) == want and all(r() is not None for r in structs.values()), structs
    ctx.sync()
    gc.collect()
    assert all(r() is None for r in structs.values())


def test_kept_outputs_given_as_a_list_are_those_of_each_call(ra, monkeypatch):
    """Another tensor put into the list is the one that the next call writes."""
    monkeypatch.setattr(ra, "_dptr", lambda t: ctypes.c_void_p(t.data_ptr()))
    wit = list(ra.witness_outputs(4, 8, "cpu"))
    bufs = {"C": torch.empty((4, 8), dtype=torch.int64), "wit": wit}
    for i in range(5):
        o = ra._outputs(4, 8, "cpu", bufs)
        assert o is ra._outputs(4, 8, "cpu", bufs)
        assert [p.value for p in o.ptr] == [x.data_ptr() for x in (bufs["C"], *bufs["wit"])]
        wit[i] = torch.empty_like(wit[i])
        bufs["wit"] = wit
    assert [p.value for p in ra._outputs(4, 8, "cpu", bufs).ptr[1:]] == [x.data_ptr() for x in wit]
