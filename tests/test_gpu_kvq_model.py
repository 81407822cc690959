"""GPU: layer steps, prompts and generation over an 8-bit cache."""
import numpy as np
import pytest

import kvq_plain
from paper_2506_03700_amd import synth
from tolerances import REG, check_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ad():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    from paper_2506_03700_amd import binding
    binding.lib()
    return binding


GQA = synth.TINY_GQA.with_(tied_head=False, vocab=640)
SHAPES = [synth.TINY.with_(tied_head=False), GQA, GQA.with_(name="tiny-gqa-bf16", dtype=synth.BF16), GQA.with_(name="tiny-gqa-f16", dtype=synth.F16),
          synth.LLAMA8B_LAYER, synth.TINY_BF16.with_(name="wide-group", n_q_heads=20, n_kv_heads=1, n_layers=2, exit_layers=(), tied_head=False)]


def as_f64(a, dtype):
    return (synth.bf16_bits_to_f32(a) if dtype == synth.BF16 else a).astype(np.float64)


def layer(s, w, l, x, pos, K, V):
    """Layer l (1-based) over rows x at pos with the attention reading K, V [n, kv heads, dh]: (output, keys, values of the rows before they are stored)."""
    W = lambda n: as_f64(w[f"layers.{l - 1}.{n}"], s.dtype)
    rms = lambda a, g: a / np.sqrt((a * a).mean(-1, keepdims=True) + s.rms_eps) * g
    m, dh, half = len(pos), s.head_dim, s.head_dim // 2
    ang = np.asarray(pos, dtype=np.float64)[:, None, None] * s.rope_base ** (-2.0 * np.arange(half) / dh)
    rot = lambda a: np.concatenate([a[..., :half] * np.cos(ang) - a[..., half:] * np.sin(ang), a[..., :half] * np.sin(ang) + a[..., half:] * np.cos(ang)], -1)
    n = rms(x, W("attn_norm"))
    q = rot((n @ W("wq").T).reshape(m, s.n_q_heads, dh))
    k = rot((n @ W("wk").T).reshape(m, s.n_kv_heads, dh))
    v = (n @ W("wv").T).reshape(m, s.n_kv_heads, dh)
    o, _ = kvq_plain.attend(q, K, V, pos)
    x = x + o @ W("wo").T
    n = rms(x, W("ffn_norm"))
    a, b = n @ W("w_gate").T, n @ W("w_up").T
    return x + (a / (1 + np.exp(-a)) * b) @ W("w_down").T, k, v


def check_stored(dtype, got, x, what):
    """Stored values against vectors x in 64 bits: equal, or a neighbouring code (a step of 2^-3 of the value, or 2^-9 of the scale, or a scale of twice the size)
    where the vector's own error crosses the border between two; few of those."""
    want = kvq_plain.values(x)
    scale = np.exp2(kvq_plain.exponents(x))[..., None]
    err = REG[dtype] * np.max(np.abs(x))
    assert np.all(np.abs(got - x) <= 2.0 ** -4 * np.abs(x) * (1 + 2.0 ** -3) + 2.0 ** -9 * scale + 2 * err), what
    # an error of err crosses one of the borders, 2^-3 of a value apart, for that share of the entries (small ones have borders 2^-9 of the scale apart)
    share = np.mean(np.abs(got - want) > 1e-6 * np.abs(want))
    limit = np.mean(np.minimum(1.0, 2 * err / np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -9 * scale))) + 3 / np.sqrt(x.size)
    assert share <= limit, f"{what}: {share:.3%} of the entries differ, {limit:.3%} expected at most"


@pytest.mark.parametrize("s", SHAPES, ids=lambda s: s.name)
def test_layer_steps(ad, s):
    """Rows of a step are stored as the definition says, and attend to what is stored, the row itself included."""
    w = synth.make_weights(s, seed=2, norm_jitter=0.2)
    g = ad.Model(s, w, max_pos=700, kvq=True)
    rng = np.random.default_rng(8)
    for ctx, m in [(0, 1), (0, 8), (1, 3), (63, 2), (60, 8), (511, 1), (530, 5), (600, 8)]:
        print(f"case {s.name} ctx={ctx} m={m}", flush=True)
        l = s.n_layers
        if ctx:
            k, v = (rng.standard_normal((ctx, s.n_kv_heads, s.head_dim)).astype(np.float32) for _ in range(2))
            g.kv_fill(l, k, v)
        g.kv_set_len(l, ctx)
        x = rng.standard_normal((m, s.d_model)).astype(np.float32)
        h = g.torch.from_numpy(x).to("cuda:0")
        pos = ctx + np.arange(m)
        g.ad_layer_step(l, h, pos)
        assert g.kv_len(l) == ctx + m
        K, V = g.kv_read(l, ctx + m)
        if ctx:
            np.testing.assert_array_equal(K[:ctx], kvq_plain.values(k))
            np.testing.assert_array_equal(V[:ctx], kvq_plain.values(v))
        want, k_own, v_own = layer(s, w, l, x.astype(np.float64), pos, K, V)
        check_stored(s.dtype, K[ctx:], k_own, "keys")
        check_stored(s.dtype, V[ctx:], v_own, "values")
        check_rows(s.dtype, h.cpu().numpy(), want, f"rows after {ctx} positions")
    g.close()


@pytest.mark.parametrize("s", SHAPES[:4], ids=lambda s: s.name)
def test_rows_of_one_call_and_of_several(ad, s):
    """Deferred rows that join later, all at once, leave the cache that one step per row leaves (up to codes next to a border)."""
    g = ad.Model(s, synth.make_weights(s, seed=3), max_pos=64, kvq=True)
    toks = np.arange(3, 11)
    for l0 in (1,):
        h = g.ad_embed(toks)
        g.ad_layer_step(l0, h, np.arange(8))
        a, codes = g.kv_read(l0, 8), h.cpu().numpy()
        g.kv_truncate(0)
        rows = []
        for i in range(8):
            h1 = g.ad_embed(toks[i:i + 1])
            g.ad_layer_step(l0, h1, [i])
            rows.append(h1.cpu().numpy())
        b = g.kv_read(l0, 8)
        for x, y in zip(a, b):
            assert np.mean(x != y) <= 0.01 and np.max(np.abs(x - y)) <= 2.0 ** -3 * np.max(np.abs(x))
        check_rows(s.dtype, codes, np.concatenate(rows), "rows")
    g.close()


ODD = GQA.with_(name="odd-bf16", dtype=synth.BF16, n_q_heads=6, n_kv_heads=2, d_model=208, d_ffn=200, n_layers=3, exit_layers=(1,), rope_base=500000.0)


@pytest.mark.parametrize("s", [ODD, ODD.with_(name="odd-f16", dtype=synth.F16), ODD.with_(name="dh128", n_q_heads=4, n_kv_heads=1, head_dim=128, d_model=256, d_ffn=688),
                               synth.TINY.with_(tied_head=False)], ids=lambda s: s.name)
def test_prompts(ad, s):
    """A prompt pass leaves what layer steps of 8 rows leave; so does a cache without the pass's scratch, and one of fp32 weights, which has none."""
    w = synth.make_weights(s, seed=4, norm_jitter=0.2)
    g = ad.Model(s, w, max_pos=1400, kvq=True)
    for n in (2, 9, 10, 33, 64, 65, 66, 129, 200, 257, 1024, 1025, 1026, 1300):
        print(f"case {s.name} {n} tokens", flush=True)
        p = synth.make_prompt(s, n, n)
        g.kv_storage.zero_()                                  # (the rotary table as well: made again)
        g.L.ad_kv_destroy(g.kv)
        ad._check(g.L.ad_kvq_create(g.model, g.kv_storage.data_ptr(), g.kv_storage.numel(), 1400, None, ad.C.byref(g.kv)))
        g.ad_generate(p, 1, 2.0, 0)
        assert g.kv_lens() == [n] * s.n_layers
        got = [g.kv_read(l, n) for l in range(1, s.n_layers + 1)]
        h = g.ad_embed([7])
        g.ad_layer_steps(1, s.n_layers, h, [n])
        row = h.cpu().numpy()
        g.kv_truncate(0)
        for i in range(0, n, 8):
            t = p[i:i + 8]
            h = g.ad_embed(t)
            for l in range(1, s.n_layers + 1):
                g.ad_layer_step(l, h, i + np.arange(len(t)))
        for l, x in enumerate(got, 1):
            for a, b in zip(x, g.kv_read(l, n)):
                # codes next to a border may fall either way, and what differs in one layer moves the next one's
                top = np.abs(b).max(axis=-1, keepdims=True)
                assert np.all(np.abs(a - b) <= 2.0 ** -3 * np.abs(b) * 1.01 + 2.0 ** -6 * top), f"layer {l}"
                assert np.mean(a != b) <= 0.02 * l, f"layer {l}: {np.mean(a != b):.3%} of the entries differ"
        h = g.ad_embed([7])
        g.ad_layer_steps(1, s.n_layers, h, [n])
        # (2 % of the codes off by 2^-3 of their value at most move a mean over the positions by far less than the stated 16-bit bar)
        want = h.cpu().numpy()
        assert np.max(np.abs(row - want)) <= 2e-2 * np.max(np.abs(want))
    g.close()


def test_storage_without_the_prompt_scratch(ad):
    """256 bytes less than ad_kvq_bytes() is a cache all the same, whose prompts go through 8 rows at a time."""
    s = ODD
    w = synth.make_weights(s, seed=4, norm_jitter=0.2)
    g = ad.Model(s, w, max_pos=300, kvq=True)
    p = synth.make_prompt(s, 7, 200)
    want, _, _ = g.ad_generate(p, 8, 2.0, 0)
    g.L.ad_kv_destroy(g.kv)
    ad._check(g.L.ad_kvq_create(g.model, g.kv_storage.data_ptr(), g.kv_storage.numel() - 256, 300, None, ad.C.byref(g.kv)))
    g.kv_storage[-(1 << 16):].fill_(0xA5)
    got, _, _ = g.ad_generate(p, 8, 2.0, 0)
    assert bool((g.kv_storage[-(1 << 16):] == 0xA5).all())
    assert len(got) == len(want) == 8
    core = 3 * ((2 * 2 * 320 * 65 + 255) // 256 * 256)
    assert g.L.ad_kvq_create(g.model, g.kv_storage.data_ptr(), core, 300, None, ad.C.byref(ad.C.c_void_p())) == ad.AD_ENOMEM
    g.close()


@pytest.mark.parametrize("s", [synth.TINY.with_(tied_head=False, vocab=512, exit_layers=(1, 2, 3)), GQA, GQA.with_(name="tiny-gqa-bf16", dtype=synth.BF16),
                               GQA.with_(name="tiny-gqa-f16", dtype=synth.F16)], ids=lambda s: s.name)
def test_generation_emits_what_plain_decoding_emits(ad, s):
    """Early exits, wrong drafts, rollbacks and deferred rows over an 8-bit cache against one token at a time over one: the same tokens, unless two logits tie."""
    g = ad.Model(s, synth.make_weights(s, seed=0, with_T=True, T_std=0.03), max_pos=160, kvq=True)
    p = synth.make_prompt(s, 0)
    n_new = 60
    plain, _, _ = g.ad_generate(p, n_new, 2.0, 0)
    K, V = g.kv_read(1, len(p) + n_new - 1)
    rejected = early = 0
    for seed in range(4):
        forced = synth.make_forced_schedule(s, seed, 160, probs=[0.6 / len(s.exit_layers)] * len(s.exit_layers))
        script = np.full(160, -1, dtype=np.int32)
        script[[40, 47, 61]] = [1, 2, 3]
        toks, st, _ = g.ad_generate(p, n_new, 0.9, 5, forced_exit=forced, scripted_draft=script)
        rejected += st["rejections"]
        early += st["early_preds"]
        assert st["bytes_algorithmic"] > 0
        same = int(np.argmin(np.append(toks == plain, False)))
        if same < n_new:
            # the logits after the common part, from a run of layer steps: the two tokens must be as good as tied
            seq = np.concatenate([p, plain[:same]])
            g.kv_truncate(0)
            for i in range(0, len(seq), 8):
                h = g.ad_embed(seq[i:i + 8])
                g.ad_layer_steps(1, s.n_layers, h, i + np.arange(len(seq[i:i + 8])))
            z = g.ad_head_logits(s.n_layers, h)[-1].cpu().numpy()
            assert abs(z[toks[same]] - z[plain[same]]) < 1e-2, (seed, same)
            continue
        k2, v2 = g.kv_read(1, len(p) + n_new - 1)
        assert np.mean(K != k2) <= 0.01 and np.mean(V != v2) <= 0.01
    assert early > 40 and rejected > 5
    # sampled decoding runs over it too
    u = synth.make_uniforms(s, 1, 160)
    toks, st, _ = g.ad_generate(p, 24, 0.0, 5, temperature=0.3, uniforms=u)
    assert len(toks) == 24 and st["early_preds"] > 0
    g.close()


def test_refusals(ad):
    import torch
    s = GQA.with_(dtype=synth.BF16)
    w = synth.make_weights(s, seed=0)
    g, other = ad.Model(s, w, max_pos=32, kvq=True, m_max=4), ad.Model(s, w, max_pos=32)
    k = torch.zeros((2, s.n_kv_heads, s.head_dim), device="cuda:0")
    q = torch.zeros((1, s.n_q_heads, s.head_dim), device="cuda:0")

    def status(f):
        with pytest.raises(ad.AdError) as e:
            f()
        return e.value.status

    assert status(lambda: g.ad_kvq_append(1, k, k, 1)) == ad.AD_ESTATE                 # not at the cache's end
    assert status(lambda: g.ad_kvq_append(0, k, k, 0)) == ad.AD_ERANGE
    assert status(lambda: g.ad_kvq_append(s.n_layers + 1, k, k, 0)) == ad.AD_ERANGE
    assert status(lambda: g.ad_kvq_append(1, k[:0], k[:0], 0)) == ad.AD_EINVAL         # (an empty tensor has no address)
    assert status(lambda: g.ad_kvq_append(1, k, k, -1)) == ad.AD_ERANGE
    g.kv_set_len(1, 31)
    assert status(lambda: g.ad_kvq_append(1, k, k, 31)) == ad.AD_ERANGE                # beyond max_pos
    g.kv_set_len(1, 0)
    assert status(lambda: g.ad_kvq_attend(1, q, [0])) == ad.AD_ERANGE                  # an empty cache
    assert status(lambda: g.ad_kvq_read(1, 0, 1)) == ad.AD_ERANGE
    g.ad_kvq_append(1, k, k, 0)
    assert status(lambda: g.ad_kvq_attend(1, q, [2])) == ad.AD_ERANGE
    assert status(lambda: g.ad_kvq_attend(1, q, [-1])) == ad.AD_ERANGE
    assert status(lambda: g.ad_kvq_attend(2, q, [0])) == ad.AD_ERANGE
    assert status(lambda: g.ad_kvq_attend(1, q.expand(5, -1, -1).contiguous(), [0] * 5)) == ad.AD_ERANGE       # more rows than m_max
    assert status(lambda: g.ad_kvq_read(1, 1, 2)) == ad.AD_ERANGE
    assert status(lambda: g.ad_kvq_read(1, 0, 0)) == ad.AD_EINVAL                      # (likewise)
    assert status(lambda: other.ad_kvq_append(1, k, k, 0)) == ad.AD_ESTATE             # a 16-bit cache
    assert status(lambda: other.ad_kvq_attend(1, q, [0])) == ad.AD_ESTATE
    L, P = g.L, ad.C.c_void_p
    st = ad._stream_ptr(torch)
    args = lambda kp, ld: (g.model, g.kv, 1, P(kp), P(k.data_ptr()), ld, 2, 2, st)
    assert L.ad_kvq_append(*args(k.data_ptr() + 4, s.d_kv)) == ad.AD_EINVAL            # alignment
    assert L.ad_kvq_append(*args(k.data_ptr(), s.d_kv + 2)) == ad.AD_EINVAL
    assert L.ad_kvq_append(*args(k.data_ptr(), s.d_kv - 4)) == ad.AD_EINVAL
    assert L.ad_kvq_append(g.model, g.kv, 1, P(k.data_ptr()), P(k.data_ptr()), s.d_kv, 2, 0, st) == ad.AD_ERANGE
    assert L.ad_kvq_append(other.model, g.kv, 1, P(k.data_ptr()), P(k.data_ptr()), s.d_kv, 2, 2, st) == ad.AD_EINVAL
    assert g.kv_lens() == [2] + [0] * (s.n_layers - 1) and set(other.kv_lens()) == {0}
    g.ad_set_layer_mode(ad.AD_LAYER_FUSED)
    h = g.ad_embed([1])
    assert status(lambda: g.ad_layer_step(1, h, [2])) == ad.AD_ESTATE
    assert status(lambda: g.ad_generate(np.arange(3, 20), 2, 0.9, 2)) == ad.AD_ESTATE
    assert g.kv_len(1) == 2
    g.ad_set_layer_mode(ad.AD_LAYER_KERNELS)
    g.ad_layer_step(1, h, [2])
    g.close()
    other.close()
