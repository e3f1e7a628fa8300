"""The gated product and the scaled token embedding as layers (ra_gate_prove,
ra_embed_prove) through the C ABI: every transcript word and table bit-exact
against the oracle over sizes around the kernels' edges, types, strides and
tokens; both together in a language model's chain of layers, verified; the
refusals.  All outputs are integers, so every comparison is exact."""
import ctypes

import numpy as np
import pytest
import torch

from helpers import pack_planes
from oracle import oracle as orc
from paper_2505_17623_amd import inputs

pytestmark = pytest.mark.gpu
P61 = (1 << 61) - 1
REST = ["t", "P", "c0", "r_claim", "rm_claim", "y_claim", "z_claim", "range_sum", "rs_evals", "bits_claim", "zc_evals",
        "r_at", "y_at"]
GATE, EMBED = ["gate_evals", "a_at", "b_at"] + REST, ["mm_evals", "a_star", "b_star"] + REST


@pytest.fixture(scope="module")
def ra():
    from paper_2505_17623_amd import ra as ra_mod
    ra_mod.lib()
    assert torch.cuda.is_available()
    return ra_mod


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def same(got, want, keys):
    bad = [k for k in keys if got["transcript"][k] != want[k]]
    assert not bad, bad
    for k in ("C", "R", "Y", "Z"):
        assert np.array_equal(got[k].cpu().numpy().astype(np.int64), want[k]), k
    assert np.array_equal(got["Rm"].cpu().numpy().view(np.uint16).astype(np.int64), want["Rm"])
    assert np.array_equal(got["bits"].cpu().numpy().view(np.uint64), pack_planes(want["bits"]))


def ints(rng, shape, dtype, top):
    x = rng.integers(-top, top, shape)
    x.reshape(-1)[:1] = -top
    return x.astype(dtype)


# --- the gated product ---------------------------------------------------------
SHAPES = [(1, 1), (1, 2), (2, 1), (4, 4), (1, 512), (64, 16), (1, 2048), (2048, 1), (4, 1024), (64, 128), (256, 64),
          (8, 4096), (256, 256), (512, 256)]


@pytest.mark.parametrize("n,k", SHAPES)
@pytest.mark.parametrize("relu,mode", [(False, 0), (True, 1)])
def test_gate_matches_oracle(ra, n, k, relu, mode):
    rng = np.random.default_rng(n + 7 * k)
    A, B = ints(rng, (n, k), np.int32, 1 << 14), ints(rng, (n, k), np.int32, 1 << 13)
    chal = inputs.xorshift64_stream(100 + n + k, 1000)
    want = orc.prove_gate_layer(A, B, 9, relu, mode, chal, 0)
    ctx = ra.Context(chal)
    got = ra.prove_gate(ctx, dev(A), dev(B), 9, relu, mode)
    same(got, want, GATE)
    assert ctx.cursor() == want["cursor"]


@pytest.mark.parametrize("da,db", [(np.int16, np.int16), (np.int16, np.int32), (np.int32, np.int16)])
@pytest.mark.parametrize("n,k", [(2, 8), (32, 256)])
def test_gate_types(ra, da, db, n, k):
    rng = np.random.default_rng(k)
    A, B = (ints(rng, (n, k), d, 1 << 15) for d in (da, db))
    chal = inputs.xorshift64_stream(41, 1000)
    same(ra.prove_gate(ra.Context(chal), dev(A), dev(B), 12), orc.prove_gate_layer(A, B, 12, False, 0, chal, 0), GATE)


def test_gate_extreme_values(ra):
    """The ends of int32 against small factors (the largest product is 7 2^30,
    R = 7 2^26 with s = 4: between 2^28 and 2^29, so t = 28), and rows of zeros."""
    A = np.array([[-2 ** 31, 2 ** 31 - 1, 0, 1], [2 ** 31 - 1, -2 ** 31, 5, 0], [0, 0, 0, 0], [7, -7, 2, -2]] * 512)
    B = np.array([[1, 1, 9, -2 ** 31], [-1, 1, 0, 3], [0, 0, 0, 0], [2 ** 30, 2 ** 30, -2 ** 31, 0]] * 512)
    A, B = A.astype(np.int32), B.astype(np.int32)
    chal = inputs.xorshift64_stream(43, 1000)
    want = orc.prove_gate_layer(A, B, 4, False, 0, chal, 0)
    assert want["t"] == 28
    same(ra.prove_gate(ra.Context(chal), dev(A), dev(B), 4), want, GATE)
    with pytest.raises(ra.RAError) as e:  # R past int32
        ra.prove_gate(ra.Context(chal), dev(A), dev(A), 4)
    assert e.value.code in (-3, -9)


@pytest.mark.parametrize("n,k,ld,off", [(4, 8, 8, 1), (16, 128, 200, 3), (64, 64, 129, 0), (128, 64, 64, 2)])
def test_gate_strides_and_offsets(ra, n, k, ld, off):
    """Halves of one wide tensor, rows at odd strides, unaligned bases; C and the outputs' buffers as given."""
    rng = np.random.default_rng(ld)
    wide = ints(rng, off + n * ld + k, np.int32, 1 << 12)
    d = dev(wide)
    A = torch.as_strided(d, (n, k), (ld, 1), off)
    B = torch.as_strided(d, (n, k), (ld, 1), off + min(k // 2, ld - 1))
    chal = inputs.xorshift64_stream(47, 1000)
    want = orc.prove_gate_layer(A.cpu().numpy(), B.cpu().numpy(), 8, True, 0, chal, 0)
    before = d.clone()
    same(ra.prove_gate(ra.Context(chal), A, B, 8, True), want, GATE)
    assert torch.equal(d, before)


@pytest.mark.parametrize("n,k", [(8, 4), (256, 128)])
def test_gate_broadcast_row(ra, n, k):
    """A learned scale: one row for all (stride 0), on either side, and on both."""
    rng = np.random.default_rng(n)
    A, row = ints(rng, (n, k), np.int32, 1 << 14), ints(rng, (1, k), np.int16, 1 << 12)
    chal = inputs.xorshift64_stream(53, 1000)
    r = dev(row).expand(n, k)
    full = np.broadcast_to(row, (n, k))
    want = orc.prove_gate_layer(A, full, 10, False, 0, chal, 0)
    same(ra.prove_gate(ra.Context(chal), dev(A), r, 10), want, GATE)
    want = orc.prove_gate_layer(full, A, 10, False, 0, chal, 0)
    same(ra.prove_gate(ra.Context(chal), r, dev(A), 10), want, GATE)
    want = orc.prove_gate_layer(full, full, 10, False, 0, chal, 0)
    same(ra.prove_gate(ra.Context(chal), r, r, 10), want, GATE)


# --- the embedding -----------------------------------------------------------
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (2, 1, 3), (1, 2, 1), (4, 3, 5), (1, 1000, 64), (32, 1024, 16),
                                       (64, 1025, 8), (128, 5003, 30), (1, 4097, 300), (1024, 33, 7), (256, 300, 129),
                                       (16, 40000, 24)])
@pytest.mark.parametrize("relu,mode", [(False, 0), (True, 1)])
def test_embed_matches_oracle(ra, n, vocab, d, relu, mode):
    rng = np.random.default_rng(vocab + d)
    tok = rng.integers(-1, vocab, n).astype(np.int32)
    tok[0] = vocab - 1
    E = ints(rng, (vocab, d), np.int16, 1 << 15)
    chal = inputs.xorshift64_stream(200 + n + vocab, 1000)
    want = orc.prove_embed_layer(tok, E, 1234, 8, relu, mode, chal, 0)
    ctx = ra.Context(chal)
    same(ra.prove_embed(ctx, dev(tok), dev(E), 1234, 8, relu, mode), want, EMBED)
    assert ctx.cursor() == want["cursor"]


@pytest.mark.parametrize("which", ["one", "none", "two"])
def test_embed_repeated_and_absent_tokens(ra, which):
    """Every position the same token (its weight sums all of eq(r1, .)), padding only, two tokens."""
    rng = np.random.default_rng(5)
    n, vocab, d = 2048, 500, 12
    tok = {"one": np.full(n, 321), "none": np.full(n, -1), "two": np.where(rng.random(n) < 0.3, 0, 499)}[which]
    tok = tok.astype(np.int32)
    E = ints(rng, (vocab, d), np.int16, 1 << 15)
    chal = inputs.xorshift64_stream(61, 1000)
    want = orc.prove_embed_layer(tok, E, -(2 ** 12), 9, False, 0, chal, 0)
    same(ra.prove_embed(ra.Context(chal), dev(tok), dev(E), -(2 ** 12), 9), want, EMBED)


@pytest.mark.parametrize("scale", [0, 1, -1, 2 ** 31 - 1, -(2 ** 31)])
def test_embed_scales(ra, scale):
    rng = np.random.default_rng(9)
    tok, E = rng.integers(0, 77, 16).astype(np.int32), ints(rng, (77, 16), np.int16, 1 << 11)
    chal = inputs.xorshift64_stream(67, 1000)
    want = orc.prove_embed_layer(tok, E, scale, 13, False, 0, chal, 0)
    same(ra.prove_embed(ra.Context(chal), dev(tok), dev(E), scale, 13), want, EMBED)


@pytest.mark.parametrize("vocab,d,ld,off", [(100, 16, 24, 0), (100, 16, 17, 1), (37, 5, 8, 3), (2000, 64, 64, 4)])
def test_embed_table_strides(ra, vocab, d, ld, off):
    rng = np.random.default_rng(ld)
    wide = ints(rng, off + vocab * ld, np.int16, 1 << 14)
    E = torch.as_strided(dev(wide), (vocab, d), (ld, 1), off)
    tok = rng.integers(-1, vocab, 64).astype(np.int32)
    chal = inputs.xorshift64_stream(71, 1000)
    want = orc.prove_embed_layer(tok, E.cpu().numpy(), 999, 8, False, 0, chal, 0)
    same(ra.prove_embed(ra.Context(chal), dev(tok), E, 999, 8), want, EMBED)


# --- modes of use ------------------------------------------------------------
def test_planned_deferred_repeated(ra):
    """t given, buffers kept, outputs deferred, three requests in a row on one
    stream of challenges; with and without the announced witness; the
    workspace the caller's."""
    rng = np.random.default_rng(3)
    n, k, vocab = 32, 64, 700
    A, B = ints(rng, (n, k), np.int32, 1 << 12), ints(rng, (n, k), np.int32, 1 << 12)
    tok, E = rng.integers(0, vocab, n).astype(np.int32), ints(rng, (vocab, k), np.int16, 1 << 11)
    chal = inputs.xorshift64_stream(79, 4000)
    want, cur = [], 0
    for _ in range(3):
        e = orc.prove_embed_layer(tok, E, 300, 8, False, 0, chal, cur, 16)
        g = orc.prove_gate_layer(A, B, 8, True, 0, chal, e["cursor"], 17)
        want.append((e, g))
        cur = g["cursor"]
    size = max(ra.gate_workspace_size(n, k), ra.embed_workspace_size(n, vocab, k))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    for plan in (True, False):
        for deferred in (True, False):
            ctx = ra.Context(chal, deferred=deferred)
            for e, g in want:
                ge = ra.prove_embed(ctx, dev(tok), dev(E), 300, 8, t=16, plan=plan, ws=ws)
                gg = ra.prove_gate(ctx, dev(A), dev(B), 8, True, t=17, plan=plan, ws=ws)
                if deferred:
                    ctx.sync()
                same(ge, e, EMBED)
                same(gg, g, GATE)
            assert ctx.cursor() == cur


def test_two_contexts_on_two_streams(ra):
    """Two callers at once, each on its own stream with kept buffers: the results of each alone."""
    rng = np.random.default_rng(13)
    n, k, vocab = 128, 512, 3000
    A, B = ints(rng, (n, k), np.int32, 1 << 12), ints(rng, (n, k), np.int32, 1 << 12)
    tok, E = rng.integers(0, vocab, n).astype(np.int32), ints(rng, (vocab, k), np.int16, 1 << 11)
    dA, dB, dt, dE = dev(A), dev(B), dev(tok), dev(E)
    torch.cuda.synchronize()

    def calls(seed, stream):
        with torch.cuda.stream(stream):
            ctx = ra.Context(seed=seed, stream=stream, deferred=True)
            out = []
            for _ in range(3):
                out.append(ra.prove_gate(ctx, dA, dB, 8, t=17))
                out.append(ra.prove_embed(ctx, dt, dE, 300, 8, t=16))
        return ctx, out
    alone = []
    for seed in (5, 6):
        ctx, out = calls(seed, torch.cuda.Stream())
        ctx.sync()
        alone.append([(o["transcript"], o["Z"].clone()) for o in out])
    torch.cuda.synchronize()
    both = [calls(seed, torch.cuda.Stream()) for seed in (5, 6)]
    for (ctx, out), a in zip(both, alone):
        ctx.sync()
        for o, (tr, Z) in zip(out, a):
            assert o["transcript"] == tr and torch.equal(o["Z"], Z)


@pytest.mark.parametrize("n,vocab,d,hidden,ts", [(1, 50, 12, 16, None), (8, 300, 30, 64, None), (64, 1500, 64, 256, (15, 15, 15, 21, 28, 28))])
def test_language_model_chain(ra, n, vocab, d, hidden, ts):
    """Tokens -> scaled embedding -> gated block -> logits, against the oracle
    layer by layer, and accepted by the verifier with every link named; a
    changed token or table is rejected.  Given t: |Z| <= 500 600 / 256 < 2^11
    after the embedding, |G|, |U| <= 64 2^11 90 / 256 < 2^16, so the gated
    product's R < 2^32 / 2^8, within [-2^22, 2^22) for t = 21 as 26370^2 / 256
    < 2^22."""
    rng = np.random.default_rng(n + d)
    k, s, seed = 1 << (d - 1).bit_length(), 8, 1000 + n
    tok = rng.integers(0, vocab, n).astype(np.int32)
    if n > 1:
        tok[-1] = -1
    E = ints(rng, (vocab, d), np.int16, 500)
    Wg, Wu = (ints(rng, (k, hidden), np.int16, 90) for _ in range(2))
    Wd, Wo = ints(rng, (hidden, k), np.int16, 90), ints(rng, (k, 32), np.int16, 90)
    ctx = ra.Context(seed=seed, deferred=ts is not None)
    ts, known = (ts or [-1] * 6), ts is not None
    e = ra.prove_embed(ctx, dev(tok), dev(E), 600, s, t=ts[0])
    block = ra.prove_gated_ffn(ctx, e["Z"], dev(Wg), dev(Wu), s, Wd=dev(Wd), ts=ts[1:5] if known else None)
    logits = ra.prove_layer(ctx, block[-1]["Z"], dev(Wo), s, False, t=ts[5])
    if known:
        ctx.sync()
    chal = inputs.xorshift64_stream(seed, 4000)
    we = orc.prove_embed_layer(tok, E, 600, s, False, 0, chal, 0, ts[0])
    wg = orc.prove_layer(we["Z"], Wg, s, True, 0, chal, we["cursor"], ts[1])
    wu = orc.prove_layer(we["Z"], Wu, s, False, 0, chal, wg["cursor"], ts[2])
    wm = orc.prove_gate_layer(wg["Z"], wu["Z"], s, False, 0, chal, wu["cursor"], ts[3])
    wd = orc.prove_layer(wm["Z"], Wd, s, False, 0, chal, wm["cursor"], ts[4])
    wo = orc.prove_layer(wd["Z"], Wo, s, False, 0, chal, wd["cursor"], ts[5])
    for got, want, keys in zip([e, *block, logits], (we, wg, wu, wm, wd, wo), (EMBED, EMBED, EMBED, GATE, EMBED, EMBED)):
        same(got, want, keys)

    def host(r, **more):
        return dict({x: r[x].cpu().numpy() for x in ("Z", "R", "Rm", "Y", "bits")}, transcript=r["transcript"], **more)
    z = [r["Z"].cpu().numpy() for r in [e, *block]]
    layers = [host(e, tokens=tok, B=E, scale=600), host(block[0], A=z[0], B=Wg, from_a=0),
              host(block[1], A=z[0], B=Wu, from_a=0), host(block[2], A=z[1], B=z[2], from_a=1, from_b=2),
              host(block[3], A=z[3], B=Wd, from_a=3), host(logits, A=z[4], B=Wo, from_a=4)]
    assert ra.ra_verify(seed, layers) == (0, 0)
    other = tok.copy()
    other[0] = (other[0] + 1) % vocab
    assert ra.ra_verify(seed, [dict(layers[0], tokens=other), *layers[1:]]) == (3, 0)
    table = E.copy()
    table[tok[0], 0] += 1
    assert ra.ra_verify(seed, [dict(layers[0], B=table), *layers[1:]]) == (3, 0)
    assert ra.ra_verify(seed, [*layers[:3], dict(layers[3], from_a=2, from_b=1), *layers[4:]]) == (14, 3)


def test_refusals(ra):
    chal = inputs.xorshift64_stream(83, 400)
    A = torch.full((4, 8), 9, dtype=torch.int32).cuda()
    C = torch.empty((4, 8), dtype=torch.int64).cuda()
    tok = torch.zeros(4, dtype=torch.int32).cuda()
    E = torch.full((10, 8), 9, dtype=torch.int16).cuda()
    L, p = ra.lib(), lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    ctx = ra.Context(chal)
    ev = (ctypes.c_uint64 * 64)()
    pr, mm = ra.GateProof(evals=ev), ra.MatmulProof(evals=ev)

    def gate(a=p(A), ad=2, lda=8, b=p(A), bd=2, ldb=8, n=4, k=8, c=p(C), ws=None, wb=0, out=pr):
        return L.ra_gate_prove(ctx.h, a, ad, lda, b, bd, ldb, n, k, c, ws, wb, ctypes.byref(out))

    def embed(t=p(tok), n=4, e=p(E), lde=8, vocab=10, d=8, scale=3, c=p(C), ws=None, wb=0, out=mm):
        return L.ra_embed_prove(ctx.h, t, n, e, lde, vocab, d, scale, c, ws, wb, ctypes.byref(out))
    for bad in (dict(a=None), dict(b=None), dict(c=None), dict(ad=3), dict(bd=5), dict(lda=7), dict(ldb=1), dict(n=3),
                dict(k=0), dict(out=ra.GateProof())):
        assert gate(**bad) == -1, bad
    assert gate(n=1 << 16, k=1 << 16, lda=1 << 16, ldb=1 << 16) == -9
    assert gate(ws=p(C), wb=64) == -8
    for bad in (dict(t=None), dict(e=None), dict(c=None), dict(n=0), dict(n=6), dict(lde=7), dict(vocab=0), dict(d=0),
                dict(out=ra.MatmulProof())):
        assert embed(**bad) == -1, bad
    assert embed(vocab=(1 << 22) + 1) == -9 and embed(d=(1 << 20) + 1, lde=1 << 21) == -9
    assert embed(ws=p(C), wb=64) == -8
    assert ctx.cursor() == 0
    # a token outside the vocabulary: refused, nothing consumed, and the context goes on
    for v in (10, -2, 2 ** 31 - 1, -(2 ** 31)):
        bad = tok.clone()
        bad[2] = v
        with pytest.raises(ra.RAError) as e:
            ra.prove_embed(ctx, bad, E, 3, 4)
        assert e.value.code == -1 and ctx.cursor() == 0
    want = orc.prove_embed_layer(tok.cpu().numpy(), E.cpu().numpy(), 3, 4, False, 0, chal, 0)
    same(ra.prove_embed(ctx, tok, E, 3, 4), want, EMBED)
    # the order of a layer's calls; no gather link after such a layer
    with pytest.raises(ra.RAError) as e:
        ra.link_prove(ctx, A, torch.zeros(4, dtype=torch.int32).cuda())
    assert e.value.code == -7
    assert gate() == 0
    assert gate() == -7 and embed() == -7
    # a range given too small
    ctx = ra.Context(chal)
    with pytest.raises(ra.RAError) as e:
        ra.prove_gate(ctx, A * 1000, A * 1000, 4, t=2)
    assert e.value.code == -4
    # challenges that run out, and a transcript context
    ctx = ra.Context(chal[:5])
    assert gate() == -5 and embed() == -5
    ctx = ra.Context(fs_domain=bytes(32))
    assert gate() == -5 and embed() == -5


def test_deferred_bad_token_is_reported_at_sync(ra):
    tok = torch.tensor([0, 99], dtype=torch.int32).cuda()
    E = torch.ones((10, 8), dtype=torch.int16).cuda()
    ctx = ra.Context(seed=4, deferred=True)
    ra.prove_embed(ctx, tok, E, 3, 4, t=10)
    with pytest.raises(ra.RAError) as e:
        ctx.sync()
    assert e.value.code == -1


def test_deferred_bad_token_found_in_a_later_layer(ra):
    """The first wait is a later layer's (its witness finds t): it reports the
    refusal and is itself done, and the context goes on from there."""
    rng = np.random.default_rng(18)
    A, B = (ints(rng, s, np.int16, 300) for s in ((8, 16), (16, 8)))
    chal = inputs.xorshift64_stream(91, 1000)
    ctx = ra.Context(chal, deferred=True)
    ra.prove_embed(ctx, dev(np.array([0, 99], dtype=np.int32)), dev(np.ones((10, 8), dtype=np.int16)), 3, 4, t=10)
    start = ctx.cursor()
    want = orc.prove_layer(A, B, 8, True, 0, chal, start)
    C, mm = ra.ra_sumcheck_matmul_prove(ctx, dev(A), dev(B))
    here, outs = ctx.cursor(), ra.witness_outputs(8, 8, "cuda")
    assert here > start
    with pytest.raises(ra.RAError) as e:
        ra.ra_rescale_relu_witness(ctx, C, 8, True, outs=outs)
    assert e.value.code == -1 and ctx.cursor() == here
    R, _, Y, _, bits = outs
    rg = ra.ra_range_prove(ctx, bits, R, Y, ra.WitnessInfo(s=8, relu=1, round_mode=0, t=want["t"], P=want["P"]))
    ctx.sync()
    assert mm["mm_evals"] == want["mm_evals"] and rg["rs_evals"] == want["rs_evals"]


def test_refused_layers_spend_their_announced_witness(ra):
    """A witness announced for a layer whose product call is refused (a bad
    token, a bad argument) is not made by the next layer: the announced buffers
    stay as they are, and the next layer is the oracle's."""
    rng = np.random.default_rng(17)
    A, B = (ints(rng, s, np.int16, 300) for s in ((64, 64), (64, 64)))
    E = dev(ints(rng, (50, 16), np.int16, 300))
    chal = inputs.xorshift64_stream(89, 1000)
    want = orc.prove_layer(A, B, 8, True, 0, chal, 0)
    for refused in ("token", "argument"):
        ctx, outs = ra.Context(chal), ra.witness_outputs(64, 64, "cuda")
        for o in outs:
            o.fill_(77)
        ra.ra_witness_plan(ctx, 8, True, 0, want["t"], outs)
        with pytest.raises(ra.RAError) as e:
            if refused == "token":
                ra.ra_embed_prove(ctx, dev(np.full(256, 50, dtype=np.int32)), E, 3)
            else:
                ra.ra_gate_prove(ctx, dev(A[:3]), dev(A[:3]))
        assert e.value.code == -1 and ctx.cursor() == 0
        torch.cuda.synchronize()
        if refused == "token":  # that layer's own witness is in them; what counts is the next layer's
            for o in outs:
                o.fill_(77)
        res = ra.prove_layer(ctx, dev(A), dev(B), 8, True, t=want["t"], plan=False)
        same(res, want, EMBED)
        assert all(bool((o == 77).all()) for o in outs)


@pytest.mark.parametrize("n,k", [(1, 2), (64, 512), (128, 1024)])
def test_gate_t_given_at_its_edge(ra, n, k):
    """t given: the least t that holds R is taken, one less is refused, past
    and below the 2^18 at which the claims' sums change (t = 17 and 18), and a
    refused layer leaves the context usable for its witness alone."""
    rng = np.random.default_rng(n)
    chal = inputs.xorshift64_stream(97, 1000)
    for bits in (11, 17, 18, 21, 28):
        A = ints(rng, (n, k), np.int32, 1 << bits)
        B = ints(rng, (n, k), np.int32, 16)
        want = orc.prove_gate_layer(A, B, 4, False, 0, chal, 0)
        t = want["t"]
        same(ra.prove_gate(ra.Context(chal), dev(A), dev(B), 4, t=t), want, GATE)
        with pytest.raises(ra.RAError) as e:
            ra.prove_gate(ra.Context(chal), dev(A), dev(B), 4, t=t - 1)
        assert e.value.code == -4


def test_embed_wide_range(ra):
    """R past 2^18 with t given (the claims' sums reduced a row at a time), many rows a thread."""
    rng = np.random.default_rng(23)
    n, vocab, d = 8192, 64, 256
    tok, E = rng.integers(0, vocab, n).astype(np.int32), ints(rng, (vocab, d), np.int16, 1 << 15)
    chal = inputs.xorshift64_stream(101, 1000)
    want = orc.prove_embed_layer(tok, E, 2 ** 19 + 1, 6, False, 0, chal, 0)
    assert want["t"] > 18
    same(ra.prove_embed(ra.Context(chal), dev(tok), dev(E), 2 ** 19 + 1, 6, t=want["t"]), want, EMBED)


def test_large_products_with_and_without_the_announcement(ra):
    """2^22 outputs, where a thread takes four rows of an embedding at a time
    and a gated product has four passes: the announced witness (made with the
    product) and the witness call's own give the same proof and tables."""
    rng = np.random.default_rng(29)
    n, vocab, k = 8192, 999, 512
    tok, E = dev(rng.integers(-1, vocab, n).astype(np.int32)), dev(ints(rng, (vocab, k - 3), np.int16, 1 << 11))
    A, B = (dev(ints(rng, (n, k), np.int32, 1 << 12)) for _ in range(2))
    got = []
    for plan in (True, False):
        ctx = ra.Context(seed=31)
        got.append((ra.prove_embed(ctx, tok, E, 4000, 8, t=18, plan=plan), ra.prove_gate(ctx, A, B, 8, t=18, plan=plan)))
    for x, y in zip(*got):
        assert x["transcript"] == y["transcript"]
        assert all(torch.equal(x[key], y[key]) for key in ("C", "R", "Rm", "Y", "Z", "bits"))


@pytest.mark.parametrize("n,m,k", [(1, 1, 1), (1, 64, 8), (1, 4096, 64), (2, 2048, 256), (8, 32, 32), (32, 512, 128),
                                   (2, 64, 4096), (2, 64, 8192), (1, 128, 16384),
                                   (64, 64, 64)])
@pytest.mark.parametrize("kind", ["int16", "int32", "int24"])
def test_matrix_layers_of_few_rows(ra, n, m, k, kind):
    """A block's projections for few tokens: the inner dimension split in a
    workgroup (to 32 rows and 4096 columns), beside sizes past that; int32
    inputs with four limbs and with three; t found, given and announced."""
    rng = np.random.default_rng(n + m + k)
    A = ints(rng, (n, m), np.int16, 2000) if kind == "int16" else \
        ints(rng, (n, m), np.int32, 1 << 20) if kind == "int32" else np.abs(ints(rng, (n, m), np.int32, 1 << 20))
    A.flat[0] = {"int16": -2000, "int32": -(1 << 24), "int24": (1 << 24) - 1}[kind]
    B = ints(rng, (m, k), np.int16, 300)
    chal = inputs.xorshift64_stream(93, 1000)
    for relu, mode in ((True, 0), (False, 1)):
        want = orc.prove_layer(A, B, 12, relu, mode, chal, 0)
        for t, plan in ((-1, False), (want["t"], False), (want["t"], True)):
            ctx = ra.Context(chal)
            same(ra.prove_layer(ctx, dev(A), dev(B), 12, relu, mode, t, plan=plan), want, EMBED)


def test_gated_block_refused_leaves_the_context_as_its_calls_do(ra):
    """A block whose gated product has t = 39 (R past int32: not implemented): the refusal, the
    mode and the position are those of the same calls made one by one."""
    rng = np.random.default_rng(19)
    X = ints(rng, (8, 64), np.int32, 1 << 21)
    Wg, Wu = (ints(rng, (64, 32), np.int16, 300) for _ in range(2))
    one, block = ra.Context(seed=8), ra.Context(seed=8)
    gate = ra.prove_layer(one, dev(X), dev(Wg), 8, True)
    up = ra.prove_layer(one, dev(X), dev(Wu), 8, False)
    codes = []
    for call in (lambda: ra.prove_gate(one, gate["Z"], up["Z"], 8),
                 lambda: ra.prove_gated_ffn(block, dev(X), dev(Wg), dev(Wu), 8)):
        with pytest.raises(ra.RAError) as e:
            call()
        codes.append(e.value.code)
    assert codes == [-9, -9] and not block.deferred and one.cursor() == block.cursor()
    for ctx in (one, block):  # the layer waits for its witness, as after any refused range
        with pytest.raises(ra.RAError) as e:
            ra.prove_gate(ctx, gate["Z"], up["Z"], 8)
        assert e.value.code == -7


@pytest.mark.parametrize("down", [False, True])
def test_gated_block_without_t_equals_its_calls(ra, down):
    """t found: the block, which waits once a layer, and its calls one by one, twice in a row."""
    rng = np.random.default_rng(20)
    X = ints(rng, (8, 64), np.int16, 500)
    Wg, Wu = (ints(rng, (64, 128), np.int16, 60) for _ in range(2))
    Wd = dev(ints(rng, (128, 64), np.int16, 60)) if down else None
    X, Wg, Wu = dev(X), dev(Wg), dev(Wu)
    one, block = ra.Context(seed=9), ra.Context(seed=9)
    for _ in range(2):
        gate, up = ra.prove_layer(one, X, Wg, 8, True), ra.prove_layer(one, X, Wu, 8, False)
        want = [gate, up, ra.prove_gate(one, gate["Z"], up["Z"], 8)]
        if down:
            want.append(ra.prove_layer(one, want[2]["Z"], Wd, 8, False))
        got = ra.prove_gated_ffn(block, X, Wg, Wu, 8, Wd=Wd)
        assert not block.deferred and one.cursor() == block.cursor() and len(got) == len(want)
        for x, y in zip(got, want):
            assert x["transcript"] == y["transcript"] and x["transcript"]["rs_evals"]
            assert all(torch.equal(x[key], y[key]) for key in ("C", "R", "Rm", "Y", "Z", "bits"))


def test_an_announcement_does_not_outlive_a_refusal(ra):
    """A layer given up before its product call, by a check in Python, by a
    refused matrix call or by hand, leaves nothing to the next layer: the kept
    outputs stay as they are, and the next layer, whose witness is not
    announced, is the oracle's."""
    rng = np.random.default_rng(33)
    A, B = (ints(rng, (64, 64), np.int16, 300) for _ in range(2))
    dA, dB = dev(A), dev(B)
    E, I = dev(ints(rng, (50, 64), np.int16, 300)), dev(ints(rng, (64, 64), np.int32, 300))  # noqa: E741
    chal = inputs.xorshift64_stream(103, 1000)
    want = orc.prove_layer(A, B, 8, True, 0, chal, 0)
    t = want["t"]
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    for how in ("tokens", "shape", "matrix", "workspace", "withdrawn"):
        ctx, bufs = ra.Context(chal), {"C": torch.empty((64, 64), dtype=torch.int64, device="cuda")}
        bufs["wit"] = outs = ra.witness_outputs(64, 64, "cuda")
        for o in outs:
            o.fill_(77)
        if how == "withdrawn":
            ra.ra_witness_plan(ctx, 8, True, 0, t, outs)
            L = ra.lib()
            one = ctypes.c_void_p(outs[0].data_ptr())
            assert L.ra_witness_plan(ctx.h, 8, 1, 0, t, one, None, None, None, None, 4096) == -1  # some null: refused
            assert L.ra_witness_plan(ctx.h, 0, 0, 0, -1, None, None, None, None, None, 0) == 0
        else:
            with pytest.raises((AssertionError, ra.RAError)):
                if how == "tokens":  # torch's default type
                    ra.prove_embed(ctx, torch.zeros(64, dtype=torch.int64).cuda(), E, 3, 8, True, t=t, bufs=bufs)
                elif how == "shape":
                    ra.prove_gate(ctx, I, I[:32], 8, True, t=t, bufs=bufs)
                elif how == "matrix":
                    ra.prove_layer(ctx, dA, dB[:32], 8, True, t=t, bufs=bufs)
                else:
                    ra.prove_layer(ctx, dA, dB, 8, True, t=t, bufs=bufs, ws=small)
        assert ctx.cursor() == 0
        same(ra.prove_layer(ctx, dA, dB, 8, True, t=t, plan=False), want, EMBED)
        assert all(bool((o == 77).all()) for o in outs), how


def bad_embedding(ra, ctx, vocab=10):
    """An embedding with a token outside the vocabulary, its product call alone."""
    return ra.ra_embed_prove(ctx, dev(np.array([0, vocab], dtype=np.int32)), dev(np.ones((vocab, 8), dtype=np.int16)), 3)


def go_on(ra, ctx, chal, start, seed=41):
    """The context is between layers at `start`: a matrix layer with t found, a gated one and an
    embedding with t given are the oracle's, one after the other."""
    rng = np.random.default_rng(seed)
    A, B, G = ints(rng, (8, 16), np.int16, 300), ints(rng, (16, 8), np.int16, 300), ints(rng, (8, 8), np.int32, 300)
    tok, E = rng.integers(0, 9, 4).astype(np.int32), ints(rng, (9, 8), np.int16, 300)
    assert ctx.cursor() == start
    want = [orc.prove_layer(A, B, 8, True, 0, chal, start)]
    want.append(orc.prove_gate_layer(G, G, 8, True, 0, chal, want[0]["cursor"], 12))
    want.append(orc.prove_embed_layer(tok, E, 3, 4, False, 0, chal, want[1]["cursor"], 12))
    got = [ra.prove_layer(ctx, dev(A), dev(B), 8, True), ra.prove_gate(ctx, dev(G), dev(G), 8, True, t=12),
           ra.prove_embed(ctx, dev(tok), dev(E), 3, 4, t=12)]
    ctx.sync()
    for g, w, keys in zip(got, want, (EMBED, GATE, EMBED)):
        same(g, w, keys)
    assert ctx.cursor() == want[-1]["cursor"]


@pytest.mark.parametrize("wait", ["sync", "synchronous", "binding", "profiling", "witness", "commitment"])
def test_bad_token_found_by_its_own_layers_wait(ra, wait):
    """Whatever waits between a deferred embedding's product call and its
    witness call finds the refusal: the challenges are given back, the layer's
    further calls are out of order, and later layers are the oracle's (no
    challenge is given back twice)."""
    chal = inputs.xorshift64_stream(107, 1000)
    ctx = ra.Context(chal, deferred=True)
    C, _ = bad_embedding(ra, ctx)
    assert ctx.cursor() == 8  # log n, log k, log V: 1 + 3 + 4
    code = None
    if wait == "sync":
        with pytest.raises(ra.RAError) as e:
            ctx.sync()
        code = e.value.code
    elif wait == "synchronous":
        ctx.set_deferred(False)
        ctx.set_deferred(True)
    elif wait == "binding":
        ra.ra_mle_bind(ctx, dev(np.ones((2, 2), dtype=np.int16)), True, [5])
    elif wait == "profiling":
        ctx.set_profiling(False)
    elif wait == "commitment":
        ra.commit_generators(ctx, bytes(32), 4)
    else:  # t found: the witness call waits
        with pytest.raises(ra.RAError) as e:
            ra.ra_rescale_relu_witness(ctx, C, 4, False)
        code = e.value.code
    assert ctx.cursor() == 0
    with pytest.raises(ra.RAError) as e:
        ra.ra_rescale_relu_witness(ctx, C, 4, False, t=10)
    assert e.value.code == -7
    if code is None:  # kept for the next sync, reported once
        with pytest.raises(ra.RAError) as e:
            ctx.sync()
        code = e.value.code
    assert code == -1
    ctx.sync()
    go_on(ra, ctx, chal, 0)


def test_bad_token_found_between_witness_and_range(ra):
    """The layer's range call is not enqueued yet: given back as well; enqueued, the layer stands."""
    chal = inputs.xorshift64_stream(109, 1000)
    for enqueued in (False, True):
        ctx = ra.Context(chal, deferred=True)
        C, _ = bad_embedding(ra, ctx)
        (R, _, Y, _, bits), info = ra.ra_rescale_relu_witness(ctx, C, 4, False, t=10)
        if enqueued:
            ra.ra_range_prove(ctx, bits, R, Y, info)
        start = ctx.cursor() if enqueued else 0
        with pytest.raises(ra.RAError) as e:
            ctx.sync()
        assert e.value.code == -1 and ctx.cursor() == start
        if not enqueued:
            with pytest.raises(ra.RAError) as e:
                ra.ra_range_prove(ctx, bits, R, Y, info)
            assert e.value.code == -7
        go_on(ra, ctx, chal, start)


def test_bad_token_found_when_the_pinned_area_grows(ra):
    """With the area (4096 words at first) all but full of pending outputs, a call of the
    refused layer itself waits for it to grow.  Whichever call that is, the
    layer is given back or stands, and the context goes on from its cursor."""
    chal = inputs.xorshift64_stream(113, 20000)
    rng = np.random.default_rng(43)
    G = dev(ints(rng, (1, 1), np.int32, 100))
    found = set()
    # a gated layer of one entry leaves 8 + 16 + 24 words pending (s + t + 2 = 16 planes: 4 rounds of 4 words and
    # six, rounded up to eights), 84 of them 4032; the embedding's product takes 4 + 3 log V, rounded up: 8 .. 56,
    # its witness 16 and its range call 56
    for lv in (1, 4, 6, 9, 12, 14, 17):
        ctx = ra.Context(chal, deferred=True)
        for _ in range(84):
            ra.prove_gate(ctx, G, G, 8, t=6)
        start, where = ctx.cursor(), "later"
        C, _ = bad_embedding(ra, ctx, 1 << lv)
        try:
            (R, _, Y, _, bits), info = ra.ra_rescale_relu_witness(ctx, C, 4, False, t=10)
            where = "range"
            ra.ra_range_prove(ctx, bits, R, Y, info)
            start, where = ctx.cursor(), "stands"
        except ra.RAError as e:
            assert e.code == -1 and ctx.cursor() == start
            where = "witness" if where == "later" else where
            ctx.sync()
        else:
            with pytest.raises(ra.RAError) as e:
                ctx.sync()
            assert e.value.code == -1
        found.add(where)
        go_on(ra, ctx, chal, start)
    assert {"witness", "range"} <= found, found


@pytest.mark.parametrize("n,vocab,d,ld", [(4, 16400, 70, 70), (2, 16385, 33, 35), (1, 16400, 1100, 1100), (2, 40, 1100, 1100),
                                          (1, 40, 1101, 1101), (2, 40, 2080, 2080), (1, 100, 4127, 4130)])
@pytest.mark.parametrize("t", [-1, 15])
def test_embed_wide_tables_match_oracle(ra, n, vocab, d, ld, t):
    """The table's pass past its first trip: a quarter of a row of more than
    eight chunks of 32 entries (d > 1024), a ragged last chunk or none, rows at
    odd strides, in both heights of a workgroup (two tiles of rows from 16384
    padded rows on)."""
    rng = np.random.default_rng(vocab + d)
    wide = ints(rng, (vocab, ld), np.int16, 1 << 15)
    wide[0, d - 1], wide[vocab - 1, d - 1] = -(1 << 15), (1 << 15) - 1
    E = dev(wide)[:, :d]
    tok = rng.integers(-1, vocab, n).astype(np.int32)
    tok[0] = vocab - 1
    chal = inputs.xorshift64_stream(300 + d, 1000)
    want = orc.prove_embed_layer(tok, wide[:, :d], 250, 8, False, 0, chal, 0, t)
    ctx = ra.Context(chal)
    same(ra.prove_embed(ctx, dev(tok), E, 250, 8, t=t), want, EMBED)
    assert ctx.cursor() == want["cursor"]


def eq_table(z):
    """eq(z, .) in Python integers, z's first coordinate the index's highest bit."""
    t = [1]
    for x in z:
        t = [w for v in t for w in (v * (1 - x) % P61, v * x % P61)]
    return t


def at_point(ra, ctx, T, rows, cols):
    """The multilinear extension of a device matrix at (rows, cols), by the two bindings."""
    v = ra.ra_mle_bind(ctx, T, True, rows)
    return int(ra.ra_mle_bind(ctx, v.reshape(1, -1), False, cols, field=True)[0])


def chain_end(c0, evals, deg, rho):
    """The last value of a sum-check whose every round's sum is the value before it."""
    cur = c0
    for j, x in enumerate(rho):
        g = evals[(deg + 1) * j:(deg + 1) * (j + 1)]
        assert (g[0] + g[1]) % P61 == cur, j
        cur = 0
        for a in range(deg + 1):
            num = den = 1
            for b in range(deg + 1):
                if b != a:
                    num, den = num * (x - b) % P61, den * (a - b) % P61
            cur = (cur + g[a] * num * pow(den, P61 - 2, P61)) % P61
    return cur


def check_witness_of(ra, ctx, got, C, s, relu, r1, r2):
    """The tables from C by their definitions (to nearest), the claims as the tables' extensions."""
    R, tr = (C + (1 << (s - 1))) >> s, got["transcript"]
    Rm, Y = C + (1 << (s - 1)) - (R << s), R.abs()
    Z = (R + Y) // 2 if relu else R
    assert torch.equal(got["C"], C)
    for key, x in (("R", R), ("Y", Y), ("Z", Z)):
        assert torch.equal(got[key].long(), x), key
    assert torch.equal(got["Rm"].long() & 0xFFFF, Rm)
    word = Rm + ((R + (2 << tr["t"])) << s)
    if relu:
        word += Y << (s + tr["t"] + 2)
    assert torch.equal(got["bits"].reshape(C.shape), word)
    assert tr["c0"] == at_point(ra, ctx, C, r1, r2)
    for key, x in (("r_claim", R), ("rm_claim", Rm), ("y_claim", Y), ("z_claim", Z)):
        assert tr[key] == at_point(ra, ctx, x.int(), r1, r2), key


@pytest.mark.parametrize("n,vocab,d,t,off", [(8192, 999, 509, 18, 0), (8192, 999, 509, 16, 0), (65536, 50, 126, 16, 0),
                                             (8192, 300, 251, 17, 1), (1 << 18, 7, 12, 18, 1)])
def test_embed_of_many_rows_against_its_definition(ra, n, vocab, d, t, off):
    """2^21 to 2^23 outputs, where a thread takes four rows at a time, once or
    twice, in pairs of columns or (C off by one entry) alone, the claims' sums
    reduced a row at a time (t = 18) or not."""
    rng = np.random.default_rng(n + d)
    k, s, scale, seed = 1 << (d - 1).bit_length(), 8, 4000, 71
    ln, lk, lv = n.bit_length() - 1, k.bit_length() - 1, (vocab - 1).bit_length()
    tok = rng.integers(-1, vocab, n).astype(np.int32)
    E = dev(ints(rng, (vocab, d), np.int16, 1 << 11))
    c = [int(x) for x in inputs.xorshift64_stream(seed, ln + lk + lv)]
    r1, r2, rho = c[:ln], c[ln:ln + lk], c[ln + lk:]
    ctx, help_ctx = ra.Context(seed=seed), ra.Context(seed=1)
    buf = torch.empty(n * k + off, dtype=torch.int64, device="cuda")
    bufs = {"C": buf[off:].reshape(n, k), "wit": ra.witness_outputs(n, k, "cuda")}
    dt = dev(tok)
    got = ra.prove_embed(ctx, dt, E, scale, s, t=t, bufs=bufs)
    C = torch.zeros((n, k), dtype=torch.int64, device="cuda")
    C[:, :d] = scale * E.long()[dt.long().clamp(min=0)] * (dt >= 0).long()[:, None]
    check_witness_of(ra, help_ctx, got, C, s, False, r1, r2)
    tr = got["transcript"]
    assert chain_end(tr["c0"], tr["mm_evals"], 2, rho) == tr["a_star"] * tr["b_star"] % P61
    e1, ev = eq_table(r1), eq_table(rho)
    assert tr["a_star"] == scale * sum(x * ev[v] for x, v in zip(e1, tok.tolist()) if v >= 0) % P61
    pad = torch.zeros((1 << lv, k), dtype=torch.int16, device="cuda")
    pad[:vocab, :d] = E
    assert tr["b_star"] == at_point(ra, help_ctx, pad, rho, r2)


@pytest.mark.parametrize("n,k,relu", [(512, 512, True), (8192, 512, False), (2048, 4096, True)])
def test_gate_of_many_passes_against_its_definition(ra, n, k, relu):
    """2^18, 2^22 and 2^23 entries: two, three and four passes before the last rounds."""
    rng = np.random.default_rng(n + k)
    s, seed, lN, ln = 8, 73, (n * k).bit_length() - 1, n.bit_length() - 1
    A, B = dev(ints(rng, (n, k), np.int32, 1 << 12)), dev(ints(rng, (n, k), np.int16, 1 << 11))
    c = [int(x) for x in inputs.xorshift64_stream(seed, 2 * lN)]
    r, rho = c[:lN], c[lN:]
    ctx, help_ctx = ra.Context(seed=seed), ra.Context(seed=1)
    got = ra.prove_gate(ctx, A, B, s, relu, t=15)
    check_witness_of(ra, help_ctx, got, A.long() * B.long(), s, relu, r[:ln], r[ln:])
    tr, eq = got["transcript"], 1
    for x, y in zip(r, rho):
        eq = eq * (x * y + (1 - x) * (1 - y)) % P61
    assert chain_end(tr["c0"], tr["gate_evals"], 3, rho) == eq * tr["a_at"] * tr["b_at"] % P61
    assert tr["a_at"] == at_point(ra, help_ctx, A, rho[:ln], rho[ln:])
    assert tr["b_at"] == at_point(ra, help_ctx, B, rho[:ln], rho[ln:])


def in_chunks(ra, ctx, T, rows, cols, log_chunk):
    """at_point, 2^log_chunk rows at a time."""
    hi = len(rows) - log_chunk
    step, e = 1 << log_chunk, eq_table(rows[:hi])
    return sum(w * at_point(ra, ctx, T[i * step:(i + 1) * step], rows[hi:], cols) for i, w in enumerate(e)) % P61


def check_large_outputs(ra, ctx, outs, C, want, s, t, r1, r2, log_chunk):
    """Tables and C against want(first row, last row), in chunks, and C~."""
    R, Rm, Y, Z, bits = outs
    step = 1 << log_chunk
    for i in range(0, C.shape[0], step):
        c, j = want(i, i + step), i + step
        assert torch.equal(C[i:j], c), i
        r = (c + (1 << (s - 1))) >> s
        rm = c + (1 << (s - 1)) - (r << s)
        assert torch.equal(R[i:j].long(), r) and torch.equal(Z[i:j].long(), r) and torch.equal(Y[i:j].long(), r.abs())
        assert torch.equal(Rm[i:j].long() & 0xFFFF, rm)
        assert torch.equal(bits.reshape(C.shape)[i:j], rm + ((r + (2 << t)) << s)), i
    return in_chunks(ra, ctx, C, r1, r2, log_chunk)


def test_gate_past_32_bit_offsets(ra):
    """2^29 entries: C, the bit words and every int32 table reach past 2^31 or 2^32 bytes."""
    n, k, s, t, seed = 1 << 15, 1 << 14, 8, 15, 77
    lN, ln, part = 29, 15, 9
    g = torch.Generator(device="cuda").manual_seed(1)
    A = torch.randint(-4096, 4096, (n, k), dtype=torch.int32, device="cuda", generator=g)
    B = torch.randint(-1024, 1024, (n, k), dtype=torch.int16, device="cuda", generator=g)
    outs = ra.witness_outputs(n, k, "cuda")
    ctx, help_ctx = ra.Context(seed=seed), ra.Context(seed=1)
    ra.ra_witness_plan(ctx, s, False, 0, t, outs)
    C, tr = ra.ra_gate_prove(ctx, A, B)
    _, info = ra.ra_rescale_relu_witness(ctx, C, s, False, 0, t, outs)
    c = [int(x) for x in inputs.xorshift64_stream(seed, 2 * lN)]
    r, rho = c[:lN], c[lN:]
    at = check_large_outputs(ra, help_ctx, outs, C, lambda i, j: A[i:j].long() * B[i:j].long(), s, t, r[:ln], r[ln:], part)
    assert tr["c0"] == at
    assert ((int(info.r_claim) << s) + int(info.rm_claim) - (1 << (s - 1)) - at) % P61 == 0
    assert info.rm_claim == in_chunks(ra, help_ctx, (C + (1 << (s - 1)) & ((1 << s) - 1)).int(), r[:ln], r[ln:], part)
    eq = 1
    for x, y in zip(r, rho):
        eq = eq * (x * y + (1 - x) * (1 - y)) % P61
    assert chain_end(tr["c0"], tr["gate_evals"], 3, rho) == eq * tr["a_at"] * tr["b_at"] % P61
    assert tr["a_at"] == in_chunks(ra, help_ctx, A, rho[:ln], rho[ln:], part)
    assert tr["b_at"] == in_chunks(ra, help_ctx, B, rho[:ln], rho[ln:], part)


@pytest.mark.parametrize("n,vocab,d", [(1 << 17, 300, 4096), (4, (1 << 20) + 3, 4096)])
def test_embed_past_32_bit_offsets(ra, n, vocab, d):
    """2^29 outputs; a table of 8.6 GB, its last rows among the tokens."""
    s, t, scale, seed = 8, 16, 500, 79
    ln, lk, lv = n.bit_length() - 1, 12, (vocab - 1).bit_length()
    g = torch.Generator(device="cuda").manual_seed(2)
    E = torch.randint(-(1 << 15), 1 << 15, (vocab, d), dtype=torch.int16, device="cuda", generator=g)
    tok = torch.randint(-1, vocab, (n,), dtype=torch.int32, device="cuda", generator=g)
    tok[0], tok[n - 1] = vocab - 1, vocab - 2
    outs = ra.witness_outputs(n, d, "cuda")
    ctx, help_ctx = ra.Context(seed=seed), ra.Context(seed=1)
    ra.ra_witness_plan(ctx, s, False, 0, t, outs)
    C, tr = ra.ra_embed_prove(ctx, tok, E, scale)
    _, info = ra.ra_rescale_relu_witness(ctx, C, s, False, 0, t, outs)
    c = [int(x) for x in inputs.xorshift64_stream(seed, ln + lk + lv)]
    r1, r2, rho = c[:ln], c[ln:ln + lk], c[ln + lk:]
    part = min(ln, 11)

    def want(i, j):
        v = tok[i:j].long()
        return scale * E[v.clamp(min=0)].long() * (v >= 0).long()[:, None]
    at = check_large_outputs(ra, help_ctx, outs, C, want, s, t, r1, r2, part)
    assert tr["c0"] == at
    assert ((int(info.r_claim) << s) + int(info.rm_claim) - (1 << (s - 1)) - at) % P61 == 0
    assert chain_end(tr["c0"], tr["mm_evals"], 2, rho) == tr["a_star"] * tr["b_star"] % P61
    ev = eq_table(rho)
    assert tr["a_star"] == scale * sum(x * ev[v] for x, v in zip(eq_table(r1), tok.tolist()) if v >= 0) % P61
    v = torch.zeros(1 << lv, dtype=torch.int64, device="cuda")  # e(v), from the rows in blocks of 2^14
    for i in range(0, vocab, 1 << 14):
        block = E[i:i + (1 << 14)]
        rows = 1 << (block.shape[0] - 1).bit_length()
        if rows != block.shape[0]:
            block = torch.cat([block, block.new_zeros(rows - block.shape[0], d)])
        v[i:i + rows] = ra.ra_mle_bind(help_ctx, block, False, r2)
    assert tr["b_star"] == int(ra.ra_mle_bind(help_ctx, v.reshape(-1, 1), True, rho, field=True)[0])
