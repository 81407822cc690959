"""GPU: the 8-bit cache by itself -- what is stored, what is read out, attention over it -- against the definitions in 64 bits."""
import ctypes as C

import numpy as np
import pytest

import kvq_plain
from paper_2506_03700_amd import synth

pytestmark = pytest.mark.gpu

HEADS = [(4, 4, 64), (4, 2, 64), (32, 8, 128), (5, 5, 128), (16, 1, 128), (40, 1, 64)]


@pytest.fixture(scope="module")
def ad():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2506_03700_amd import binding
    binding.lib()
    return binding


def small(Hq, Hkv, dh, dtype=synth.BF16, **kw):
    return synth.TINY.with_(name="kvq", n_layers=2, exit_layers=(), d_model=64, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=dh, d_ffn=64, vocab=64, dtype=dtype, **kw)


def model(ad, heads, max_pos, dtype=synth.BF16):
    s = small(*heads, dtype=dtype)
    return ad.Model(s, synth.make_weights(s, seed=0), max_pos, kvq=True)


def rows(rng, n, Hkv, dh):
    """Keys and values of different sizes, with vectors at the edges of the scale's choice."""
    x = rng.standard_normal((2, n, Hkv, dh)) * np.exp2(rng.integers(-6, 7, (2, n, Hkv, 1)))
    edge = [0.0, 448.0, np.nextafter(np.float32(448), np.float32(1e9)), 447.0, 1.75, 1.7500001, 2.0 ** -118, 2.0 ** -130, 1e-42, 3.4028235e38, 2.0 ** 127]
    for i, e in enumerate(edge):
        at = rng.integers(0, n), rng.integers(0, Hkv)
        x[(i % 2,) + at] = np.clip(x[(i % 2,) + at], -1, 1) * e
        x[(i % 2,) + at + (rng.integers(0, dh),)] = e * (1 if i % 3 else -1)
    return x.astype(np.float32)


def dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda:0")


@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_store_and_read_out(ad, heads):
    """Codes and scales bit for bit, for starts and lengths at the edges of blocks; nothing else in the storage changes."""
    import torch
    Hq, Hkv, dh = heads
    g = model(ad, heads, 300)
    rng = np.random.default_rng(sum(heads))
    for pos0, n in [(0, 1), (0, 64), (0, 300), (63, 1), (63, 2), (64, 63), (1, 200), (64, 128), (17, 47), (299, 1), (128, 172)]:
        print(f"case {heads} pos0={pos0} n={n}", flush=True)
        k, v = rows(rng, n, Hkv, dh)
        g.kv_storage.fill_(0xA5)
        g.kv_set_len(2, pos0)
        before = g.kv_storage.clone()
        g.ad_kvq_append(2, dev(k), dev(v), pos0)
        assert g.kv_len(2) == pos0 + n and g.kv_len(1) == 0
        kr, vr = (x.cpu().numpy().astype(np.float64) for x in g.ad_kvq_read(2, pos0, n))
        # (read out as fp32 holds it: entries from 248 * 2^120 on round to 256 * 2^120 = 2^128, which fp32 does not have)
        with np.errstate(over="ignore"):
            np.testing.assert_array_equal(kr, kvq_plain.values(k).astype(np.float32))
            np.testing.assert_array_equal(vr, kvq_plain.values(v).astype(np.float32))
        Kc, Vc, Ks, Vs = g.kvq_views()
        at = slice(pos0, pos0 + n)
        np.testing.assert_array_equal(Ks[1, :, at].cpu().numpy().T, kvq_plain.exponents(k) + 127)
        np.testing.assert_array_equal(Vs[1, :, at].cpu().numpy().T, kvq_plain.exponents(v) + 127)
        # the codes are the format's own: as torch reads them
        code = Kc[1, :, at].contiguous().view(torch.float8_e4m3fn).float().permute(1, 0, 2).cpu().numpy().astype(np.float64)
        np.testing.assert_array_equal(code * np.exp2(kvq_plain.exponents(k))[..., None], kvq_plain.values(k))
        # everything outside the rows is as it was
        mask = torch.ones_like(g.kv_storage, dtype=torch.bool)
        now, g.kv_storage = g.kv_storage, mask.to(torch.uint8)
        mk, mv, mks, mvs = g.kvq_views()
        mk[1, :, at] = mks[1, :, at] = mvs[1, :, at] = 0
        by_pos = mv[1].permute(0, 1, 3, 2)                       # [kv head][block][position][dim]
        for p in range(pos0, pos0 + n):
            by_pos[:, p // 64, p % 64] = 0
        mask, g.kv_storage = g.kv_storage.bool(), now
        assert torch.equal(now[mask], before[mask])
    g.close()


def test_entries_that_are_no_numbers(ad):
    g = model(ad, (4, 2, 64), 64)
    rng = np.random.default_rng(1)
    k, v = rows(rng, 9, 2, 64)
    k[0, 0, 3], k[0, 1, 5], v[2, 0, 7], v[4, 1, :], k[5, 0, :] = np.nan, np.inf, -np.inf, np.nan, np.inf
    g.ad_kvq_append(1, dev(k), dev(v), 0)
    for got, x in zip(g.ad_kvq_read(1, 0, 9), (k, v)):
        with np.errstate(over="ignore"):
            np.testing.assert_array_equal(got.cpu().numpy(), kvq_plain.values(x).astype(np.float32))
    g.close()


def test_filling_and_reading_a_layer(ad):
    """kv_fill and kv_read, as for any cache: lengths stay, no rows are no error, a refusal changes nothing."""
    g = model(ad, (4, 2, 64), 70)
    k, v = rows(np.random.default_rng(2), 70, 2, 64)
    g.kv_set_len(1, 70)
    g.kv_fill(1, k, v)
    g.kv_fill(1, k[:0], v[:0])
    assert g.kv_len(1) == 70 and g.kv_len(2) == 0
    with np.errstate(over="ignore"):
        for got, x in zip(g.kv_read(1, 70), (k, v)):
            np.testing.assert_array_equal(got, kvq_plain.values(x).astype(np.float32))
    assert all(x.shape == (0, 2, 64) for x in g.kv_read(1, 0))
    with pytest.raises(ad.AdError) as e:
        g.kv_fill(1, *rows(np.random.default_rng(3), 71, 2, 64))
    assert e.value.status == ad.AD_ERANGE and g.kv_len(1) == 70
    g.close()


def test_rows_further_apart(ad):
    """ld beyond the rows' own width: what lies between is neither read nor written."""
    import torch
    g = model(ad, (4, 2, 64), 200)
    rng = np.random.default_rng(2)
    k, v = rows(rng, 100, 2, 64)
    P = C.c_void_p
    wide = torch.full((2, 100, 148), float("nan"), device="cuda:0")
    wide[0, :, :128], wide[1, :, :128] = dev(k).reshape(100, 128), dev(v).reshape(100, 128)
    s = P(torch.cuda.current_stream().cuda_stream)
    assert g.L.ad_kvq_append(g.model, g.kv, 1, P(wide[0].data_ptr()), P(wide[1].data_ptr()), 148, 0, 100, s) == 0
    out = torch.full((2, 50, 132), 7.0, device="cuda:0")
    assert g.L.ad_kvq_read(g.model, g.kv, 1, 31, 50, P(out[0].data_ptr()), P(out[1].data_ptr()), 132, s) == 0
    out = out.cpu().numpy()
    assert np.all(out[:, :, 128:] == 7.0)
    for o, x in zip(out, (k, v)):
        with np.errstate(over="ignore"):
            np.testing.assert_array_equal(o[:, :128].reshape(50, 2, 64), kvq_plain.values(x)[31:81].astype(np.float32))
    g.close()


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("ctx", [1, 2, 47, 64, 65, 256, 513, 777, 2111])
def test_attention(ad, heads, ctx):
    """Rows in any order of positions, the first and the last among them; what lies behind the cache's end may be anything."""
    Hq, Hkv, dh = heads
    g = model(ad, heads, ctx + 70)
    g.kv_storage.fill_(0xFF)                                     # codes that are no numbers, scales beyond all
    rng = np.random.default_rng(ctx + dh)
    k = rng.standard_normal((ctx, Hkv, dh)).astype(np.float32)
    v = (rng.standard_normal((ctx, Hkv, dh)) * np.exp2(rng.integers(-9, 4, (ctx, Hkv, 1)))).astype(np.float32)
    g.ad_kvq_append(1, dev(k), dev(v), 0)
    kq, vq = kvq_plain.values(k), kvq_plain.values(v)
    for m in (1, 2, 5, 8):
        pos = rng.integers(0, ctx, m)
        if m > 1:
            pos[0], pos[-1] = ctx - 1, 0
        if m == 1 or m == 8:
            pos = np.maximum(0, ctx - m + np.arange(m))          # the newest ones
        q = (rng.standard_normal((m, Hq, dh)) * np.exp2(rng.integers(-3, 3, (m, Hq, 1)))).astype(np.float32)
        q[m - 1, Hq - 1] = 0.0                                   # every key alike
        print(f"case {heads} ctx={ctx} pos={list(pos)}", flush=True)
        out = g.ad_kvq_attend(1, dev(q), pos).cpu().numpy()
        want, bound = kvq_plain.attend(q, kq, vq, pos)
        assert np.all(np.abs(out - want) <= bound), np.max(np.abs(out - want) / bound)
    g.close()


def test_attention_of_extreme_sizes(ad):
    """Values and queries near both ends of the range of fp32, next to ordinary ones; one key that takes all the weight."""
    heads = Hq, Hkv, dh = 8, 2, 128
    g = model(ad, heads, 512)
    rng = np.random.default_rng(3)
    n = 300
    k = rng.standard_normal((n, Hkv, dh)).astype(np.float32)
    v = rng.standard_normal((n, Hkv, dh)).astype(np.float32)
    v[7] *= np.float32(1e30)
    v[100:] *= np.float32(1e-30)
    k[200, 0] *= 30.0
    g.ad_kvq_append(1, dev(k), dev(v), 0)
    kq, vq = kvq_plain.values(k), kvq_plain.values(v)
    q = rng.standard_normal((4, Hq, dh)).astype(np.float32)
    q[0] *= np.float32(1e-35)
    q[1] *= np.float32(20.0)
    for pos in ([299, 299, 299, 6], [6, 150, 64, 255]):
        out = g.ad_kvq_attend(1, dev(q), pos).cpu().numpy()
        want, bound = kvq_plain.attend(q, kq, vq, pos)
        # (values 2^-40 and less of the largest that a block has are below what a probability holds: off by 2^-38 of that largest)
        floor = np.array([np.abs(vq[: p + 1]).max() * 2.0 ** -37 for p in pos])[:, None]
        assert np.all(np.abs(out - want) <= bound + floor)
    # a row of queries that is not finite is no number and leaves the others alone
    ok = g.ad_kvq_attend(1, dev(q), [299] * 4).cpu().numpy()
    q[2, 3, 5] = np.inf
    out = g.ad_kvq_attend(1, dev(q), [299] * 4).cpu().numpy().reshape(4, Hq, dh)
    assert np.all(np.isnan(out[2, 3]))
    out[2, 3] = ok.reshape(4, Hq, dh)[2, 3]
    np.testing.assert_array_equal(out, ok.reshape(4, Hq, dh))
    g.close()


@pytest.mark.parametrize("heads", [(32, 8, 128), (4, 2, 64), (8, 8, 128)], ids=str)
def test_entries_that_are_no_numbers_reach_only_rows_that_see_them(ad, heads):
    Hq, Hkv, dh = heads
    ctx = 331
    g = model(ad, heads, ctx)
    rng = np.random.default_rng(4)
    k, v = (rng.standard_normal((ctx, Hkv, dh)).astype(np.float32) for _ in range(2))
    q = rng.standard_normal((8, Hq, dh)).astype(np.float32)
    pos = ctx - 8 + np.arange(8)
    g.ad_kvq_append(1, dev(k), dev(v), 0)
    ok = g.ad_kvq_attend(1, dev(q), pos).cpu().numpy().reshape(8, Hq, dh)
    for t in (0, 3, 7):
        for what in (0, 1):
            k2, v2 = k.copy(), v.copy()
            (v2 if what else k2)[ctx - 8 + t, Hkv - 1, 17] = np.nan
            g.kv_truncate(0)
            g.ad_kvq_append(1, dev(k2), dev(v2), 0)
            out = g.ad_kvq_attend(1, dev(q), pos).cpu().numpy().reshape(8, Hq, dh)
            G = Hq // Hkv
            hit = out[t:, Hq - G:, 17] if what else out[t:, Hq - G:]
            assert np.all(np.isnan(hit))
            clean = out.copy()
            clean[t:, Hq - G:] = ok[t:, Hq - G:]                 # (rows that see it and heads that share it)
            if what:
                assert np.all(np.isfinite(np.delete(out, 17, axis=2)))
            # the others: the same but for the scale of the vector that is no number, which is a weight of 0 here
            want, bound = kvq_plain.attend(q, kvq_plain.values(k), kvq_plain.values(v), pos)
            assert np.all(np.abs(clean.reshape(8, -1) - want) <= bound)
    g.close()


def test_the_same_rows_leave_the_same_cache(ad):
    """In one call, in pieces, and after rollbacks of other rows."""
    import torch
    heads = Hq, Hkv, dh = 4, 2, 64
    g = model(ad, heads, 400)
    rng = np.random.default_rng(5)
    k, v = rows(rng, 333, Hkv, dh)
    kd, vd = dev(k), dev(v)
    g.ad_kvq_append(1, kd, vd, 0)
    whole = g.kv_storage.clone()
    g.kv_storage.zero_()
    g.kv_truncate(0)
    at = 0
    while at < 333:
        n = min(333 - at, int(rng.integers(1, 70)))
        wrong = min(8, 400 - at)
        g.ad_kvq_append(1, 100.0 * vd[:wrong].contiguous(), kd[:wrong].contiguous(), at)
        g.kv_truncate(at)
        g.ad_kvq_append(1, kd[at:at + n].contiguous(), vd[at:at + n].contiguous(), at)
        at += n
    a = g.ad_kvq_read(1, 0, 333)
    g.kv_storage.copy_(whole)
    b = g.ad_kvq_read(1, 0, 333)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    g.close()


def test_repeated_and_captured(ad):
    """The same bits again, on another stream, and in a graph that is replayed over new rows with eager work in between."""
    import torch
    heads = Hq, Hkv, dh = 32, 8, 128
    ctx = 3001
    g = model(ad, heads, ctx + 8)
    rng = np.random.default_rng(6)
    data = [[dev(x) for x in (rng.standard_normal((ctx + 5, Hkv, dh)).astype(np.float32), rng.standard_normal((ctx + 5, Hkv, dh)).astype(np.float32),
                              rng.standard_normal((5, Hq, dh)).astype(np.float32))] for _ in range(4)]
    pos = ctx + np.arange(5)

    def eager(k, v, q):
        g.kv_truncate(0)
        g.ad_kvq_append(1, k, v, 0)
        return g.ad_kvq_attend(1, q, pos).clone()

    want = [eager(*d) for d in data]
    assert all(torch.equal(eager(*d), w) for d, w in zip(data, want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = [eager(*d) for d in data]
    s.synchronize()
    assert all(torch.equal(x, w) for x, w in zip(got, want))
    k, v, q = (x.clone() for x in data[0])
    g.kv_truncate(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.ad_kvq_append(1, k, v, 0)
        out = g.ad_kvq_attend(1, q, pos)
    for i in (1, 2, 3, 0, 2):
        for x, y in zip((k, v, q), data[i]):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
        assert torch.equal(g.ad_kvq_attend(1, data[i][2], pos), want[i])
        torch.cuda.synchronize()
    g.close()


def test_offsets_beyond_32_bits(ad):
    """A cache whose codes of one kind take more than 4 GiB: the last kv head's last positions."""
    import torch
    heads = Hq, Hkv, dh = 8, 8, 128
    max_pos = 4_300_000
    g = model(ad, heads, max_pos, dtype=synth.F32)
    rng = np.random.default_rng(7)
    k, v = (rng.standard_normal((9, Hkv, dh)).astype(np.float32) for _ in range(2))
    at = max_pos - 9
    g.kv_set_len(2, at)
    g.ad_kvq_append(2, dev(k), dev(v), at)
    for got, x in zip(g.ad_kvq_read(2, at, 9), (k, v)):
        np.testing.assert_array_equal(got.cpu().numpy(), kvq_plain.values(x))
    # every earlier position is zeros (a scale of 0 too): its score is 0 and its value adds nothing
    q = (8.0 * rng.standard_normal((3, Hq, dh))).astype(np.float32)
    pos = [max_pos - 1, max_pos - 4, max_pos - 9]
    out = g.ad_kvq_attend(2, dev(q), pos).cpu().numpy().reshape(3, Hq, dh)
    kq, vq = kvq_plain.values(k), kvq_plain.values(v)
    for r, p in enumerate(pos):
        see = p - at + 1
        for h in range(Hq):
            s = kq[:see, h] @ q[r, h].astype(np.float64) / np.sqrt(dh)
            top = max(0.0, s.max())
            w = np.exp(s - top)
            want = w @ vq[:see, h] / (w.sum() + at * np.exp(-top))
            size = np.max(np.abs(kq[:see, h]) @ np.abs(q[r, h])) / np.sqrt(dh)
            # chains of sums over 4.3 million weights, 264 of a lane at a time: 2^-24 * 300 on top of the scores' error
            tol = (w @ np.abs(vq[:see, h]) / (w.sum() + at * np.exp(-top))) * (np.expm1(2 * size * (2.0 ** -22 + 140 * 2.0 ** -24)) + 300 * 2.0 ** -24) + 1e-38
            assert np.all(np.abs(out[r, h] - want) <= tol)
    g.close()
