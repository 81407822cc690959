"""GPU: filtered distributions, draws from them and verification between them, against the definitions in 64 bits.

What is kept, and every token, must be the definition's unless it is decided by less than the arithmetic holds: weights are multiples of 2^-(62 - bits of
vocab) of the largest, so a sum over the vocabulary is off by less than vocab * that < 2^-27 of it for the vocabularies here (MARGIN); a
probability is off by that and its rounding to fp32."""
import ctypes as C

import numpy as np
import pytest

import filter_plain
from filter_plain import Row
from paper_2506_03700_amd import synth

pytestmark = pytest.mark.gpu

MARGIN = 2.0 ** -27
SMALL = synth.TINY.with_(name="small", tied_head=False, n_layers=1, exit_layers=(), d_model=16, n_q_heads=1, n_kv_heads=1, d_ffn=8, dtype=synth.BF16)
FILTERS = [(0, 0.0, 0.0), (1, 0.0, 0.0), (50, 0.0, 0.0), (0, 0.9, 0.0), (0, 0.0, 0.05), (50, 0.9, 0.02), (700, 0.99, 0.0), (1 << 20, 0.3, 1e-4), (3, 1.0, 1.0),
           (20000, 0.999, 0.0), (2000, 0.5, 1e-3)]


@pytest.fixture(scope="module")
def ad():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2506_03700_amd import binding
    binding.lib()
    return binding


def model(ad, V):
    s = SMALL.with_(vocab=V)
    return ad.Model(s, synth.make_weights(s, seed=0), max_pos=8)


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def logits(rng, V, kind):
    z = rng.standard_normal(V).astype(np.float32)
    if kind == "tail":
        z = (12 - 1.2 * np.log1p(rng.permutation(V)) + 0.3 * z).astype(np.float32)
    elif kind == "flat":                                             # every id alike
        z[:] = 1.25
    elif kind == "steps":                                            # a few values, many ids each; zeros of both signs
        z = np.round(z * 2).astype(np.float32) / 2
        z[z == 0] = np.where(rng.random(np.count_nonzero(z == 0)) < 0.5, 0.0, -0.0).astype(np.float32)
    elif kind == "masked":
        z = (3 * z).astype(np.float32)
        z[rng.random(V) < 0.7] = -np.inf
        z[rng.integers(0, V)] = 1.0
    elif kind == "huge":
        with np.errstate(over="ignore"):
            z = (z * np.float32(1e38)).astype(np.float32)
    elif kind == "close":                                            # values that differ in their last bits
        z = (1 + rng.integers(0, 3, V) * 2.0 ** -23).astype(np.float32)
    return z


def check_probs(got, z, f, what):
    """One row of probabilities: the kept ids, each probability, their sum."""
    want = Row(z, *f)
    if not want.fine:                                                # (the largest of many "huge" logits is infinite)
        assert np.all(np.isnan(got)), what
        return 1
    kept = got > 0
    if want.margin > MARGIN:
        # (a probability below fp32's smallest is 0 either way)
        np.testing.assert_array_equal(kept, want.p > 2.0 ** -150, err_msg=what)
        np.testing.assert_allclose(got, want.p, rtol=2.0 ** -24 + MARGIN, atol=2.0 ** -149, err_msg=what)
        return 1
    # a border that is this close may fall to either side of one id (or of ids that weigh next to nothing)
    odd = kept != (want.p > 0)
    assert want.p[odd].sum() + got[odd].sum() <= 2 * max(want.p[want.p > 0].min(), got[kept].min()) + MARGIN, what
    return 0


@pytest.mark.parametrize("V", [1, 2, 63, 301, 2047, 2048, 2049, 4097, 32016, 128256])
def test_distributions(ad, V):
    rng = np.random.default_rng(V)
    g = model(ad, V)
    sure = total = 0
    for kind in ("normal", "tail", "flat", "steps", "masked", "huge", "close"):
        for i, (k, p, mp) in enumerate(FILTERS):
            T = (1.0, 0.7, 1.6, 1e-3, 30.0)[(i + len(kind)) % 5]
            rows = 1 + (i % 3 if V < 100000 else 0)
            print(f"case V={V} {kind} T={T} top_k={k} top_p={p} min_p={mp} rows={rows}", flush=True)
            z = np.stack([logits(rng, V, kind) for _ in range(rows)])
            got = g.ad_filtered_probs(dev(z), ad.Filter(T, k, p, mp)).cpu().numpy()
            for r in range(rows):
                sure += check_probs(got[r].astype(np.float64), z[r], (T, k, p, mp), f"row {r}")
                total += 1
                assert not np.isfinite(z[r].max()) or abs(got[r].sum(dtype=np.float64) - 1) < 1e-6
    assert sure >= 0.8 * total
    g.close()


@pytest.mark.parametrize("V", [600001, 1100003])
def test_long_rows(ad, V):
    """More ids than a list of a border's bucket holds, and segments longer than a workgroup's usual ones."""
    rng = np.random.default_rng(V)
    g = model(ad, V)
    for kind, T, f in [("tail", 1.0, (0, 0.95, 0.0)), ("flat", 1.0, (77777, 0.5, 0.0)), ("close", 1.0, (V - 5, 0.0, 0.0)), ("normal", 20.0, (400000, 0.9, 0.0)),
                       ("masked", 0.5, (1000, 0.8, 1e-3))]:
        print(f"case V={V} {kind}", flush=True)
        z = logits(rng, V, kind)
        got = g.ad_filtered_probs(dev(z[None]), ad.Filter(T, *f)).cpu().numpy()[0]
        check_probs(got.astype(np.float64), z, (T, *f), kind)
        want = Row(z, T, *f)
        for u in rng.random(3):
            u = filter_plain.f32(u)
            tok, prob = g.ad_sample_filtered(dev(z), ad.Filter(T, *f), u)
            t, margin = filter_plain.draw(want.p, u)
            assert tok == t or min(margin, want.margin) < MARGIN
            assert abs(prob - want.p[tok]) <= (2.0 ** -24 + MARGIN) * want.p[tok] or want.margin < MARGIN
    g.close()


@pytest.mark.parametrize("V", [1, 301, 2048, 2049, 32016, 128256])
def test_draws(ad, V):
    rng = np.random.default_rng(V + 1)
    g = model(ad, V)
    same = total = 0
    for kind in ("normal", "tail", "flat", "steps", "masked", "huge"):
        for i, (k, p, mp) in enumerate(FILTERS):
            T = (1.0, 0.6, 1.4)[(i + len(kind)) % 3]
            z = logits(rng, V, kind)
            want = Row(z, T, k, p, mp)
            print(f"case V={V} {kind} T={T} top_k={k} top_p={p} min_p={mp}", flush=True)
            for u in (0.0, filter_plain.f32(rng.random()), 1 - 2.0 ** -24):
                tok, prob = g.ad_sample_filtered(dev(z), ad.Filter(T, k, p, mp), u)
                if not want.fine:
                    assert tok == -1 and np.isnan(prob)
                    continue
                t, margin = filter_plain.draw(want.p, u)
                assert 0 <= tok < V and z[tok] > -np.inf
                total += 1
                if min(want.margin, margin) > MARGIN or tok == t:
                    same += 1
                    assert tok == t
                    if want.margin > MARGIN:
                        assert abs(prob - want.p[t]) <= (2.0 ** -24 + MARGIN) * want.p[t]
    assert same >= 0.8 * total
    g.close()


@pytest.mark.parametrize("V", [2, 301, 2049, 32016, 128256])
def test_verification(ad, V):
    rng = np.random.default_rng(V + 2)
    g = model(ad, V)
    n_cmp = n_rej = n_all = n = 0
    for case in range(44 if V < 100000 else 22):
        m = 1 + case % 8
        T = (1.0, 0.7, 1.5)[case % 3]
        f = FILTERS[case % len(FILTERS)]
        kind = ("tail", "normal", "steps", "masked")[(case // 2) % 4]
        noise = (0.0, 0.05, 0.4, 2.0)[case % 4]
        zf = np.stack([logits(rng, V, kind) for _ in range(m)])
        with np.errstate(invalid="ignore"):
            zq = (zf[:m - 1] + noise * rng.standard_normal((m - 1, V))).astype(np.float32)
        P, Q = [Row(z, T, *f) for z in zf], [Row(z, T, *f) for z in zq]
        draft = np.array([filter_plain.draw(q.p, rng.random())[0] for q in Q], dtype=np.int32)
        if case % 7 == 3 and m > 1:
            draft[m - 2] = rng.integers(0, V)                        # a token that its distribution may not hold
        ua, ur = rng.random(m - 1).astype(np.float32), rng.random(m - 1).astype(np.float32)
        uf = filter_plain.f32(rng.random())
        print(f"case V={V} #{case} m={m} {kind} T={T} {f} noise={noise}", flush=True)
        na, nx, ratio = g.ad_verify_filtered(dev(zf), dev(zq) if m > 1 else None, draft, ad.Filter(T, *f), ua, ur, uf)
        na_w, nx_w, ratio_w, margin = filter_plain.verify(P, Q, draft, ua, ur, uf)
        assert 0 <= na <= m - 1 and 0 <= nx < V
        n += 1
        # (the rest of two near distributions is a small difference: its draws' margin counts in units of their sum)
        if margin > 16 * MARGIN:
            n_cmp += 1
            n_rej += na_w < m - 1
            n_all += na_w == m - 1 and m > 1
            assert (na, nx) == (na_w, nx_w)
            k = min(na + 1, m - 1)
            np.testing.assert_allclose(ratio[:k], ratio_w[:k].astype(np.float32), rtol=2.0 ** -24 + 2 * MARGIN)
            assert np.all(ratio[k:] == 0)
    assert n_cmp >= 0.6 * n and (V == 2 or (n_rej >= 2 and n_all >= 2))
    # identical rows: everything is accepted whatever the draws, with a ratio of exactly 1
    z = np.stack([logits(rng, V, "normal") for _ in range(5)])
    d = [int(np.argmax(r)) for r in z[:4]]
    na, nx, ratio = g.ad_verify_filtered(dev(z), dev(z[:4]), d, ad.Filter(0.8, 0, 0.9, 0.0), [1 - 2.0 ** -24] * 4, [0.5] * 4, 0.25)
    assert na == 4 and np.all(ratio == 1.0)
    assert nx == filter_plain.draw(Row(z[4], 0.8, 0, 0.9, 0.0).p, 0.25)[0]
    g.close()


def test_tokens_that_a_side_does_not_hold(ad):
    """p = 0: rejected whatever the draw, and replaced from what p has and q has not; q = 0: accepted if p holds it."""
    V = 3000
    g = model(ad, V)
    z = np.full((2, V), -5.0, dtype=np.float32)
    zq = z[:1].copy()
    z[0, [10, 2500]] = [4.0, 3.0]
    zq[0, [10, 700]] = [4.0, 3.5]
    f = ad.Filter(1.0, 2, 0.0, 0.0)
    na, nx, ratio = g.ad_verify_filtered(dev(z), dev(zq), [700], f, [0.0], [0.5], 0.5)
    assert (na, ratio[0]) == (0, 0.0) and nx in (10, 2500)
    P, Q = Row(z[0], 1.0, 2), Row(zq[0], 1.0, 2)
    assert nx == filter_plain.draw(np.maximum(P.p - Q.p, 0), 0.5)[0]
    na, nx, ratio = g.ad_verify_filtered(dev(z), dev(zq), [2500], f, [1 - 2.0 ** -24], [0.5], 0.5)
    assert na == 1 and np.isinf(ratio[0])
    na, nx, ratio = g.ad_verify_filtered(dev(z), dev(zq), [5], f, [0.0], [0.5], 0.5)
    assert (na, ratio[0]) == (0, 0.0) and nx in (10, 2500)
    g.close()


@pytest.mark.parametrize("V", [301, 5000])
def test_min_p_at_its_edges(ad, V):
    """Logits next to the border by one step of fp32, a border at the top, at and below the smallest number, and temperatures at which all weights are 1 or all but one 0."""
    g = model(ad, V)
    rng = np.random.default_rng(12)
    z = rng.standard_normal(V).astype(np.float32)
    z[7] = 5.0
    for T, mp in [(1.0, 0.05), (0.3, 0.5), (2.5, 1e-4), (1.0, 1.0), (1e30, 1.0), (1e30, 0.5), (1e-30, 1e-3), (1.0, 1e-38), (1e37, 1e-30), (40.0, 0.999999)]:
        T, mp = filter_plain.f32(T), filter_plain.f32(mp)
        x = z.copy()
        with np.errstate(over="ignore"):
            edge = np.float32(5.0 + T * np.log(mp))
        if np.isfinite(edge):
            for i, e in enumerate((edge, np.nextafter(edge, np.float32(9)), np.nextafter(edge, np.float32(-1e38)))):
                x[20 + i] = min(e, np.float32(5.0))
        x[30], x[31] = -3.0e38, -0.0
        print(f"case V={V} T={T} min_p={mp}", flush=True)
        got = g.ad_filtered_probs(dev(x[None]), ad.Filter(T, 0, 0.0, mp)).cpu().numpy()[0]
        with np.errstate(over="ignore", under="ignore"):
            w = np.exp((x.astype(np.float64) - 5.0) / T)
        # the border to the two last bits of a weight in 64 bits (the exponential's own error)
        sure, out = w >= mp * (1 + 2.0 ** -51), w < mp * (1 - 2.0 ** -51)
        assert np.all(got[sure & (w > 2.0 ** -40)] > 0) and np.all(got[out] == 0)
        tok, prob = g.ad_sample_filtered(dev(x), ad.Filter(T, 0, 0.0, mp), 1 - 2.0 ** -24)
        assert 0 <= tok < V and not out[tok] and prob > 0
    g.close()


@pytest.mark.parametrize("V", [301, 5000])
def test_rows_without_a_distribution(ad, V):
    g = model(ad, V)
    rng = np.random.default_rng(9)
    ok = rng.standard_normal(V).astype(np.float32)
    bad = []
    for x in (np.nan, np.inf):
        z = ok.copy()
        z[V - 3] = x
        bad.append(z)
    bad.append(np.full(V, -np.inf, dtype=np.float32))
    for z in bad:
        for f in (ad.Filter(0.8, 0, 0.0, 0.0), ad.Filter(0.8, 5, 0.9, 0.1)):
            tok, prob = g.ad_sample_filtered(dev(z), f, 0.5)
            assert tok == -1 and np.isnan(prob)
            p = g.ad_filtered_probs(dev(np.stack([ok, z, ok])), f).cpu().numpy()
            assert np.all(np.isnan(p[1])) and abs(p[0].sum() - 1) < 1e-6 and np.array_equal(p[0], p[2])
            na, nx, ratio = g.ad_verify_filtered(dev(np.stack([ok, z, ok])), dev(np.stack([ok, ok])), [int(np.argmax(ok))] * 2, f, [0.1] * 2, [0.5] * 2, 0.5)
            assert (na, nx) == (1, -1) and ratio[0] == 1.0 and np.isnan(ratio[1])
            na, nx, ratio = g.ad_verify_filtered(dev(np.stack([ok, z])), dev(ok[None]), [int(np.argmax(ok))], f, [0.1], [0.5], 0.5)
            assert (na, nx) == (1, -1)
            # and the next call is as if nothing had been
            assert g.ad_sample_filtered(dev(ok), f, 0.5)[0] == filter_plain.draw(Row(ok, f.temperature, f.top_k, f.top_p, f.min_p).p, 0.5)[0]
    g.close()


@pytest.mark.parametrize("V", [2049, 32016, 128256, 200001])
def test_a_small_top_k(ad, V):
    """As many ids as one kernel takes and one more, at rows where they all lie in one segment, in all of them, or are equal."""
    rng = np.random.default_rng(V + 3)
    g = model(ad, V)
    for k in (1, 64, 65, 128, 129):
        for kind in ("one segment", "every segment", "flat", "steps", "close", "few left", "tail"):
            z = logits(rng, V, kind if kind in ("flat", "steps", "close") else "tail")
            if kind == "one segment":
                z[-min(V - 2048, 200):] += np.float32(20)
            elif kind == "every segment":
                z[::max(1, V // k)] = 15
            elif kind == "few left":
                z[rng.permutation(V)[max(1, k - 2):]] = -np.inf
            for p, mp in ((0.0, 0.0), (0.8, 0.0), (0.9, 0.3)):
                print(f"case V={V} {kind} top_k={k} top_p={p} min_p={mp}", flush=True)
                f = (0.9, k, p, mp)
                got = g.ad_filtered_probs(dev(z[None]), ad.Filter(*f)).cpu().numpy()[0]
                check_probs(got.astype(np.float64), z, f, kind)
                want = Row(z, *f)
                for u in (0.0, filter_plain.f32(rng.random()), 1 - 2.0 ** -24):
                    tok, prob = g.ad_sample_filtered(dev(z), ad.Filter(*f), u)
                    t, margin = filter_plain.draw(want.p, u)
                    assert tok == t or min(margin, want.margin) < MARGIN
                    assert want.margin < MARGIN or abs(prob - want.p[tok]) <= (2.0 ** -24 + MARGIN) * want.p[tok]
    g.close()


@pytest.mark.parametrize("f", [(0.9, 300, 0.93, 0.001), (0.9, 40, 0.93, 0.001), (0.9, 0, 0.0, 0.0)], ids=["boundaries", "small-top-k", "off"])
def test_repeated_and_captured(ad, f):
    """Same bits again, from another stream, and in graphs that are replayed over new rows with eager calls in between."""
    import torch
    V, m = 32016, 4
    g = model(ad, V)
    rng = np.random.default_rng(11)
    f = ad.Filter(*f)
    rows = [dev(np.stack([logits(rng, V, "tail") for _ in range(2 * m - 1)])) for _ in range(4)]
    draft = np.array([int(rows[0][m + k].argmax()) for k in range(m - 1)], dtype=np.int32)
    ua, ur = np.full(m - 1, 0.6, np.float32), np.full(m - 1, 0.3, np.float32)

    def eager(x):
        return (g.ad_filtered_probs(x[:m].contiguous(), f), g.ad_sample_filtered(x[0], f, 0.37),
                g.ad_verify_filtered(x[:m].contiguous(), x[m:].contiguous(), draft, f, ua, ur, 0.8))

    def same(a, b):
        return torch.equal(a[0], b[0]) and a[1] == b[1] and a[2][:2] == b[2][:2] and np.array_equal(a[2][2], b[2][2])

    want = [eager(x) for x in rows]
    assert all(same(eager(x), w) for x, w in zip(rows, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert all(same(eager(x), w) for x, w in zip(rows, want))
    side.synchronize()
    x, probs = rows[0].clone(), torch.empty((m, V), device="cuda:0")
    out = torch.zeros(16, dtype=torch.int32, device="cuda:0")
    P = C.c_void_p
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = P(torch.cuda.current_stream().cuda_stream)
        at = lambda i: P(out.data_ptr() + 4 * i)
        zq = P(x.data_ptr() + 4 * m * V)
        assert g.L.ad_filtered_probs(g.model, P(x.data_ptr()), m, C.byref(f), P(probs.data_ptr()), s) == 0
        assert g.L.ad_sample_filtered(g.model, P(x.data_ptr()), C.byref(f), 0.37, at(0), at(1), s) == 0
        assert g.L.ad_verify_filtered(g.model, P(x.data_ptr()), zq, draft.ctypes.data, m, C.byref(f), ua.ctypes.data, ur.ctypes.data, 0.8, at(2), at(3), at(4), s) == 0
    for i in (1, 2, 3, 0, 2, 1):
        x.copy_(rows[i])
        graph.replay()
        torch.cuda.synchronize()
        o = out.cpu().numpy()
        got = (probs, (int(o[0]), float(o[1:2].view(np.float32)[0])), (int(o[2]), int(o[3]), o[4:4 + m - 1].view(np.float32)))
        assert same(got, want[i])
        assert same(eager(rows[3 - i]), want[3 - i])
    g.close()


def test_refusals(ad):
    import torch
    g = model(ad, 301)
    z = torch.zeros((2, 301), device="cuda:0")

    def status(f):
        with pytest.raises(ad.AdError) as e:
            f()
        return e.value.status

    nan = float("nan")
    for f in [(0.0, 0, 0, 0), (-1.0, 0, 0, 0), (nan, 0, 0, 0), (float("inf"), 0, 0, 0), (1.0, -1, 0, 0), (1.0, 0, 1.1, 0), (1.0, 0, -0.1, 0), (1.0, 0, nan, 0),
              (1.0, 0, 0, 1.1), (1.0, 0, 0, -0.1), (1.0, 0, 0, nan)]:
        f = ad.Filter(*f)
        assert status(lambda: g.ad_filtered_probs(z, f)) == ad.AD_ERANGE
        assert status(lambda: g.ad_sample_filtered(z[0], f, 0.5)) == ad.AD_ERANGE
        assert status(lambda: g.ad_verify_filtered(z, z[:1], [1], f, [0.5], [0.5], 0.5)) == ad.AD_ERANGE
    f = ad.Filter(1.0, 5, 0.0, 0.0)
    for u in (1.0, -0.1, nan):
        assert status(lambda: g.ad_sample_filtered(z[0], f, u)) == ad.AD_ERANGE
        assert status(lambda: g.ad_verify_filtered(z, z[:1], [1], f, [u], [0.5], 0.5)) == ad.AD_ERANGE
        assert status(lambda: g.ad_verify_filtered(z, z[:1], [1], f, [0.5], [u], 0.5)) == ad.AD_ERANGE
        assert status(lambda: g.ad_verify_filtered(z, z[:1], [1], f, [0.5], [0.5], u)) == ad.AD_ERANGE
    assert status(lambda: g.ad_verify_filtered(z, z[:1], [301], f, [0.5], [0.5], 0.5)) == ad.AD_ERANGE
    assert status(lambda: g.ad_verify_filtered(z, z[:1], [-1], f, [0.5], [0.5], 0.5)) == ad.AD_ERANGE
    for call in (lambda: g.ad_filtered_probs(z.cpu(), f), lambda: g.ad_sample_filtered(z[0].cpu(), f, 0.5),
                 lambda: g.ad_verify_filtered(z, z[:1].cpu(), [1], f, [0.5], [0.5], 0.5), lambda: g.ad_filtered_probs(z.double(), f)):
        with pytest.raises(AssertionError):                          # (host memory, another type)
            call()
    nine = torch.zeros((9, 301), device="cuda:0")
    assert status(lambda: g.ad_filtered_probs(nine, f)) == ad.AD_ERANGE
    assert status(lambda: g.ad_verify_filtered(nine, nine[:8], [1] * 8, f, [0.5] * 8, [0.5] * 8, 0.5)) == ad.AD_ERANGE
    g.close()


UNTIED = synth.TINY.with_(name="tiny-untied", tied_head=False, vocab=512, exit_layers=(1, 2, 3))


@pytest.mark.parametrize("kvq", [False, True], ids=["cache", "cache8"])
@pytest.mark.parametrize("dtype", [synth.F32, synth.BF16], ids=["f32", "bf16"])
def test_generation(ad, dtype, kvq):
    """Filtered sampled runs, over the model's cache and over an 8-bit one: without early exits every token is the draw from the filtered final distribution; with
    them every emitted token is one that this distribution holds; a filter that keeps one id is greedy decoding; one with nothing on is no filter."""
    s = UNTIED.with_(dtype=dtype)
    max_pos, n_new = 128, 40
    g = ad.Model(s, synth.make_weights(s, seed=0, with_T=True, T_std=0.03), max_pos, kvq=kvq)
    p = synth.make_prompt(s, 0)

    def final_logits(seq):
        """of every position, by steps of 8 rows"""
        g.kv_truncate(0)
        z = []
        for i in range(0, len(seq), 8):
            h = g.ad_embed(seq[i:i + 8])
            g.ad_layer_steps(1, s.n_layers, h, i + np.arange(len(seq[i:i + 8])))
            z.append(g.ad_head_logits(s.n_layers, h).cpu().numpy())
        return np.concatenate(z)

    T, f = 0.05, dict(top_k=12, top_p=0.9, min_p=0.01)
    u = synth.make_uniforms(s, 3, max_pos)
    # logits of another grouping of the rows are off by the storage type's rounding (and by codes of the 8-bit cache that fall on the other side of a border):
    # so is a draw this near a border, or a token this near the edge of what is kept
    near = 2e-2 if dtype == synth.F32 and not kvq else 0.2
    toks, st, _ = g.ad_generate(p, n_new, 2.0, 0, temperature=T, uniforms=u, **f)
    assert st["early_preds"] == 0 and len(toks) == n_new
    z = final_logits(np.concatenate([p, toks[:-1]]))
    n = exact = 0
    for i, t in enumerate(toks):
        row = Row(z[len(p) - 1 + i], T, f["top_k"], f["top_p"], f["min_p"])
        want, margin = filter_plain.draw(row.p, u[len(p) - 1 + i, len(s.exit_layers)])
        n += 1
        exact += t == want
        assert t == want or min(margin, row.margin) < near
    assert exact >= 0.85 * n
    early = rejected = 0
    for seed, gamma, cap in [(4, 0.0, 7), (5, 0.3, 5), (6, 0.0, 3)]:
        u = synth.make_uniforms(s, seed, max_pos)
        toks, st, ev = g.ad_generate(p, n_new, gamma, cap, temperature=T, uniforms=u, **f)
        early += st["early_preds"]
        rejected += st["rejections"]
        z = final_logits(np.concatenate([p, toks[:-1]]))
        for i, t in enumerate(toks):
            row = Row(z[len(p) - 1 + i], T, f["top_k"], f["top_p"], f["min_p"])
            assert row.p[t] > 0 or row.margin < near
        again, _, _ = g.ad_generate(p, n_new, gamma, cap, temperature=T, uniforms=u, **f)
        assert np.array_equal(again, toks)
    assert early > 20 and rejected > 2
    greedy, _, _ = g.ad_generate(p, n_new, 2.0, 0)
    one, _, _ = g.ad_generate(p, n_new, 2.0, 0, temperature=0.7, uniforms=u, top_k=1)
    assert np.array_equal(one, greedy)
    plain, _, _ = g.ad_generate(p, n_new, 0.0, 5, temperature=T, uniforms=u)
    off, _, _ = g.ad_generate(p, n_new, 0.0, 5, temperature=T, uniforms=u, top_p=1.0)
    assert np.array_equal(plain, off)
    with pytest.raises(ad.AdError) as e:
        g.ad_generate(p, n_new, 0.0, 5, temperature=T, uniforms=u, top_p=1.5)
    assert e.value.status == ad.AD_ERANGE
    with pytest.raises(ad.AdError) as e:
        g.ad_generate(p, n_new, 0.0, 5, top_k=4)                     # a filter is for sampled decoding
    assert e.value.status == ad.AD_ERANGE
    g.close()


@pytest.mark.parametrize("f", [dict(top_k=12, min_p=0.01), dict(top_k=200, top_p=0.9), dict(min_p=0.05)], ids=str)
def test_generation_with_longer_rows(ad, f):
    """A vocabulary of several segments and an 8-bit cache: plain runs draw from the filtered final distribution, runs with early exits emit what it holds, whatever is
    issued ahead."""
    s = UNTIED.with_(dtype=synth.BF16, vocab=5000)
    max_pos, n_new, T, near = 96, 24, 0.05, 0.2
    g = ad.Model(s, synth.make_weights(s, seed=0, with_T=True, T_std=0.03), max_pos, kvq=True)
    p = synth.make_prompt(s, 0, 40)
    u = synth.make_uniforms(s, 3, max_pos)
    n = exact = 0
    for gamma, cap in ((2.0, 0), (0.0, 6)):
        toks, _, _ = g.ad_generate(p, n_new, gamma, cap, temperature=T, uniforms=u, **f)
        again, _, _ = g.ad_generate(p, n_new, gamma, cap, temperature=T, uniforms=u, no_issue_ahead=True, **f)
        assert np.array_equal(toks, again) and len(toks) == n_new
        seq = np.concatenate([p, toks[:-1]])
        g.kv_truncate(0)
        for i in range(0, len(seq), 8):
            h = g.ad_embed(seq[i:i + 8])
            g.ad_layer_steps(1, s.n_layers, h, i + np.arange(len(seq[i:i + 8])))
            for j, z in enumerate(g.ad_head_logits(s.n_layers, h).cpu().numpy()):
                at = i + j - (len(p) - 1)
                if at < 0:
                    continue
                row = Row(z, T, f.get("top_k", 0), f.get("top_p", 0.0), f.get("min_p", 0.0))
                want, margin = filter_plain.draw(row.p, u[i + j, len(s.exit_layers)])
                # (logits of another grouping of the rows: a draw or an edge this near may fall to the other side)
                edge = np.sort(z)[-f["top_k"]] if "top_k" in f else np.inf
                assert row.p[toks[at]] > 0 or row.margin < near or abs(float(z[toks[at]]) - edge) < near * T
                if cap == 0:
                    n += 1
                    exact += toks[at] == want
                    assert toks[at] == want or min(margin, row.margin) < near
    # logits are off by some 2^-9, weights by 2^-9 / T = 0.04 of themselves: so is a sum of weights, and about as many draws
    assert exact >= 0.85 * n and n == n_new
    g.close()


@pytest.mark.parametrize("no_verify", [False, True])
def test_generation_without_a_distribution(ad, no_verify):
    """Final logits that are no numbers end a filtered run with an error, not with a token."""
    s = UNTIED.with_(dtype=synth.F32)
    w = synth.make_weights(s, seed=0, with_T=True, T_std=0.03)
    w["final_norm"] = np.full_like(w["final_norm"], np.nan)
    g = ad.Model(s, w, 64)
    for gamma, cap in ((2.0, 0), (0.0, 4)):
        with pytest.raises(ad.AdError) as e:
            g.ad_generate(synth.make_prompt(s, 0, 20), 8, gamma, cap, temperature=0.5, uniforms=synth.make_uniforms(s, 3, 64), top_k=12, no_verify=no_verify)
        assert e.value.status == ad.AD_ERANGE and "no distribution" in str(e.value)
    g.close()
