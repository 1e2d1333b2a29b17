"""Paged trunks of contexts that the fused passes do not take (fp32 models, heads of 128): their passes run the serving operators over the
pages.  And models with scaled rotary positions, on every path.  Against the oracle, and against the contiguous trunk's kernels."""
import numpy as np
import pytest
import torch

import ssd_inputs as I
from oracle import serve_oracle as S
from oracle import ssd_oracle as O
from tests.gpu_util import TOL, TOL_BF16_OWN_PREFILL, TOL_FUSED_BF16, dev_f32, dev_i32, kv_to_device, oracle_trunk_from_arrays, row_rel_err
from tests.test_gpu_paged import _cache, _pages_in_use, _scramble_pool

pytestmark = pytest.mark.gpu

F32 = I.ModelShape(n_layers=2, d_model=256, n_q_heads=4, n_kv_heads=4, head_dim=64, d_ffn=512, vocab=1040, dtype="f32", rope_theta=10000.0)
F32_GQA = I.ModelShape(n_layers=2, d_model=256, n_q_heads=6, n_kv_heads=2, head_dim=128, d_ffn=512, vocab=1040, dtype="f32", rope_theta=10000.0)
BF16_128 = I.ModelShape(n_layers=2, d_model=512, n_q_heads=8, n_kv_heads=2, head_dim=128, d_ffn=1024, vocab=4112, dtype="bf16",
                        rope_theta=500000.0, tie_embeddings=True)
SHAPES = {"fp32": F32, "fp32, heads of 128": F32_GQA, "bf16, heads of 128": BF16_128}


@pytest.fixture(scope="module")
def B():
    from paper_2603_03251_amd import binding
    return binding


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("batch,K,F,lens", [(3, 4, 2, [61, 3, 96]), (1, 1, 1, [1]), (2, 5, 8, [300, 33])])
def test_rounds_against_the_oracle(B, name, batch, K, F, lens):
    """Prompts of different lengths prefilled on the GPU into a scrambled pool, a teacher-forced round."""
    shape, seed = SHAPES[name], 61
    w = I.make_weights(shape, seed)
    om = O.Model.from_weights(shape, w)
    model = B.ssd_model_create(shape, w)
    max_trunk = max(lens) + 4 * (K + 1) + 40 + 32 * batch
    ctx = B.ssd_ctx_create(model, batch, K, F, max_trunk, 0, 1 + batch * (max_trunk + 31) // 32)
    try:
        assert B.ssd_ctx_views(ctx).fused_pass == 0
        _scramble_pool(B, ctx, shape, batch, seed)
        prompt = I.make_prompt(shape, batch, max(lens), seed)
        B.ssd_ctx_prefill(ctx, dev_i32(prompt), lens)
        total, free = B.ssd_ctx_kv_pages(ctx)
        assert free == total - 1 - _pages_in_use(lens)
        pending = I.make_pending(shape, batch, K, seed)
        caches = []
        for b in range(batch):
            _, trunk = O.prefill(om, prompt[b, :lens[b]])
            caches.append(O.prespeculate(om, trunk, pending[b], F, 0.0, seed=seed, row_base=b * (K + 1) * F))
        f_keys, f_toks = dev_i32(np.stack([c.keys for c in caches])), dev_i32(np.stack([c.tokens for c in caches]))
        B.ssd_ctx_set_forced(ctx, f_keys, f_toks)
        B.ssd_prespeculate(ctx, dev_i32(pending), dev_f32(np.zeros(batch, np.float32)), seed)
        B.ssd_ctx_set_forced(ctx, None, None)
        got = _cache(B, ctx)
        tol = TOL["f32"] if shape.dtype == "f32" else TOL_BF16_OWN_PREFILL
        for b in range(batch):
            e = [row_rel_err(got["glue_logits"][b], caches[b].glue_logits), row_rel_err(got["logits"][b], caches[b].logits),
                 row_rel_err(got["hidden"][b], caches[b].hidden)]
            print(f"[paged operators] {name}, seq {b}: glue {e[0]:.2e}, branches {e[1]:.2e}, hidden {e[2]:.2e}", flush=True)
            assert max(e) < tol
    finally:
        B.ssd_ctx_destroy(ctx)
        B.ssd_model_destroy(model)


@pytest.mark.parametrize("name", list(SHAPES))
def test_rounds_with_rollback_beside_the_contiguous_trunk(B, name):
    """Forced rounds with accept lengths that walk the trunks over page boundaries: the same to rounding as the contiguous trunk's kernels, and
    after each refresh the pool holds exactly the pages of the verified text; a truncation; a sequence leaves and another joins its slot; the
    pool runs dry and recovers."""
    shape, seed, batch, K, F, lens = SHAPES[name], 43, 3, 3, 2, [61, 30, 95]
    model = B.ssd_model_create(shape, I.make_weights(shape, seed))
    n_pages = 1 + _pages_in_use([n + 7 * (K + 1) for n in lens])
    plain = B.ssd_ctx_create(model, batch, K, F, 160)
    paged = B.ssd_ctx_create(model, batch, K, F, 160, 0, n_pages)
    # both sum fp32 products of the same operands in other orders; bf16 models round keys and the linear layers' operands, where a
    # difference of the last bit can become one of the operand's
    tol = TOL["f32"] if shape.dtype == "f32" else TOL_FUSED_BF16
    try:
        assert B.ssd_ctx_kv_pages(paged) == (n_pages, n_pages - 1) and B.ssd_ctx_kv_pages(plain) == (0, 0)
        _scramble_pool(B, paged, shape, batch, seed)
        prompt = I.make_prompt(shape, batch, max(lens), seed)
        for ctx in (plain, paged):
            B.ssd_ctx_prefill(ctx, dev_i32(prompt), lens)
        temps = dev_f32(np.zeros(batch, np.float32))
        rng = np.random.default_rng(seed)
        forced = dev_i32(rng.integers(0, shape.vocab, (batch, K + 1, F))), dev_i32(rng.integers(0, shape.vocab, (batch, K + 1, F, K)))
        for ctx in (plain, paged):
            B.ssd_ctx_set_forced(ctx, *forced)

        def compare(what):
            outs = []
            for ctx in (plain, paged):
                B.ssd_prespeculate(ctx, pending, temps, 3)
                outs.append(_cache(B, ctx))
            for key in ("logits", "hidden", "glue_logits"):
                assert row_rel_err(outs[1][key], outs[0][key]) < tol, (what, key)

        now = list(lens)
        for rnd in range(5):
            accepts = [K, 0, 2] if rnd == 0 else [int(a) for a in rng.integers(0, K + 1, batch)]
            pending = dev_i32(I.make_pending(shape, batch, K, seed + rnd))
            compare(rnd)
            for ctx in (plain, paged):
                B.ssd_ctx_commit(ctx, dev_i32(np.array(accepts, np.int32)))
                B.ssd_ctx_refresh_bounds(ctx)
            now = [n + a + 1 for n, a in zip(now, accepts)]
            assert B.ssd_ctx_kv_pages(paged)[1] == n_pages - 1 - _pages_in_use(now), (rnd, now)
        back = [max(1, n - 40) for n in now]
        for ctx in (plain, paged):
            B.ssd_ctx_truncate_trunk(ctx, back)
        compare("after truncation")
        for ctx in (plain, paged):
            B.ssd_ctx_truncate_trunk(ctx, back)
            B.ssd_ctx_release_sequence(ctx, 1)
            B.ssd_ctx_prefill_sequence(ctx, 1, dev_i32(prompt[2, :77]))
        compare("another prompt in slot 1")
        B.ssd_ctx_refresh_bounds(paged)
        for b in (0, 1):
            B.ssd_ctx_release_sequence(paged, b)
        with pytest.raises(B.SsdError) as err:
            for n in (140, 141, 142):
                for b in range(batch):
                    B.ssd_ctx_prefill_sequence(paged, b, dev_i32(I.make_prompt(shape, 1, n, seed)[0]))
        assert err.value.status == -4 and "out of KV pages" in str(err.value)
        for b in range(batch):
            B.ssd_ctx_release_sequence(paged, b)
        assert B.ssd_ctx_kv_pages(paged) == (n_pages, n_pages - 1)
    finally:
        B.ssd_ctx_destroy(plain)
        B.ssd_ctx_destroy(paged)
        B.ssd_model_destroy(model)


@pytest.mark.parametrize("name", list(SHAPES))
def test_loaded_and_synthetic_trunks(B, name):
    """The same stored keys through ssd_ctx_load_trunk and ssd_ctx_fill_synthetic_kv, contiguous and paged: equal to rounding, on a trunk long
    enough for several splits."""
    shape, seed, batch, K, P = SHAPES[name], 5, 2, 5, 700
    model = B.ssd_model_create(shape, I.make_weights(shape, seed))
    tol = TOL["f32"] if shape.dtype == "f32" else TOL_FUSED_BF16
    ctxs = [B.ssd_ctx_create(model, batch, K, 1, 800, 0, n) for n in (0, 60)]
    try:
        k, v = I.make_prefix_kv(shape, batch, P, seed)
        pending = dev_i32(I.make_pending(shape, batch, K, seed))
        for fill in (lambda c: B.ssd_ctx_load_trunk(c, kv_to_device(k, shape.dtype), kv_to_device(v, shape.dtype), P),
                     lambda c: B.ssd_ctx_fill_synthetic_kv(c, [P, 31], 9)):
            outs = []
            for c in ctxs:
                fill(c)
                logits = torch.empty((batch, K + 1, shape.vocab), device="cuda")
                B.ssd_ctx_extend(c, pending, 0, logits)
                one = torch.empty((batch, 1, shape.vocab), device="cuda")
                B.ssd_ctx_extend(c, pending[:, :1].contiguous(), 0, one)
                outs.append((logits.cpu().numpy(), one.cpu().numpy()))
            for a, b in zip(*outs):
                assert row_rel_err(b, a) < tol
    finally:
        for c in ctxs:
            B.ssd_ctx_destroy(c)
        B.ssd_model_destroy(model)


def test_a_trunk_beyond_16384_positions(B):
    shape, seed, K = BF16_128, 8, 2
    model = B.ssd_model_create(shape, I.make_weights(shape, seed))
    ctxs = [B.ssd_ctx_create(model, 1, K, 1, 20100, 0, n) for n in (0, 640)]
    try:
        outs = []
        for c in ctxs:
            B.ssd_ctx_fill_synthetic_kv(c, [20001], 4)
            logits = torch.empty((1, K + 1, shape.vocab), device="cuda")
            B.ssd_ctx_extend(c, dev_i32(I.make_pending(shape, 1, K, seed)), 0, logits)
            outs.append(logits.cpu().numpy())
        assert row_rel_err(outs[1], outs[0]) < TOL_FUSED_BF16
    finally:
        for c in ctxs:
            B.ssd_ctx_destroy(c)
        B.ssd_model_destroy(model)


@pytest.mark.parametrize("P", [20, 61, 300])
def test_extend_rows_of_a_paged_trunk_do_not_feel_a_later_token_without_values(B, P):
    """A token whose embedding is NaN: the rows of an extend before it keep their bits, those from it on are NaN."""
    shape, K, seed, bad = BF16_128, 5, 5 + P, 7
    w = I.make_weights(shape, seed)
    w["embed"][bad] = np.nan
    model = B.ssd_model_create(shape, w)
    ctx = B.ssd_ctx_create(model, 2, K, 1, P + 2 * K + 2, 0, 30)
    try:
        k, v = I.make_prefix_kv(shape, 2, P, seed)
        B.ssd_ctx_load_trunk(ctx, kv_to_device(k, "bf16"), kv_to_device(v, "bf16"), P)
        pending = I.make_pending(shape, 2, K, seed)
        pending[pending == bad] = bad + 1
        out = []
        for token in (bad + 2, bad):
            pending[0, 3] = token
            logits = torch.empty((2, K + 1, shape.vocab), dtype=torch.float32, device="cuda")
            B.ssd_ctx_extend(ctx, dev_i32(pending), 0, logits)
            # (the embedding is the LM head too: the token's own column is NaN everywhere)
            out.append(np.delete(logits.cpu().numpy(), bad, axis=2))
        assert np.isfinite(out[0]).all()
        assert np.array_equal(out[1][0, :3], out[0][0, :3]) and np.array_equal(out[1][1], out[0][1])
        assert np.isnan(out[1][0, 3:]).all()
    finally:
        B.ssd_ctx_destroy(ctx)
        B.ssd_model_destroy(model)


BF16_64 = I.ModelShape(n_layers=2, d_model=512, n_q_heads=8, n_kv_heads=2, head_dim=64, d_ffn=1024, vocab=4112, dtype="bf16",
                       rope_theta=500000.0, tie_embeddings=True)


@pytest.mark.parametrize("scaling,settings", [("linear", dict(factor=4.0)), ("bands", dict(factor=8.0, low=1.0, high=4.0, original=64.0)),
                                              ("ramp", dict(factor=4.0, low=1.0, high=8.0, original=256.0, magnitude=1.2))])
@pytest.mark.parametrize("name,pages,flags", [("fused", 0, 0), ("fused", 12, 0), ("fused", 0, 1), ("fp32", 0, 0), ("fp32", 12, 0),
                                              ("bf16, heads of 128", 0, 0), ("bf16, heads of 128", 12, 0)])
def test_models_with_scaled_rotary_positions(B, monkeypatch, scaling, settings, name, pages, flags):
    """ssd_model_set_rope on every path: a prompt prefilled on the GPU and a teacher-forced round against the oracle, which is given the scaled
    frequencies."""
    shape, seed, K, F, n = {**SHAPES, "fused": BF16_64}[name], 12, 3, 2, 90
    settings = dict(settings)
    magnitude = settings.pop("magnitude", 1.0)
    theta = 20000.0
    freq = S.rope_frequencies(theta, shape.head_dim, scaling, **settings)
    monkeypatch.setattr(O, "rope", lambda x, pos, _theta: S.rotate(x, np.asarray(pos), freq, "half", magnitude)[0])
    w = I.make_weights(shape, seed)
    om = O.Model.from_weights(shape, w)
    model = B.ssd_model_create(shape, w)
    B.ssd_model_set_rope(model, B.rope_config(theta, shape.head_dim, scaling=scaling, magnitude=magnitude, **settings))
    ctx = B.ssd_ctx_create(model, 1, K, F, 128, flags, pages)
    try:
        prompt = I.make_prompt(shape, 1, n, seed)
        B.ssd_ctx_prefill(ctx, dev_i32(prompt), [n])
        pending = I.make_pending(shape, 1, K, seed)
        _, trunk = O.prefill(om, prompt[0])
        want = O.prespeculate(om, trunk, pending[0], F, 0.0, seed=seed)
        f_keys, f_toks = dev_i32(want.keys[None]), dev_i32(want.tokens[None])
        B.ssd_ctx_set_forced(ctx, f_keys, f_toks)
        B.ssd_prespeculate(ctx, dev_i32(pending), dev_f32(np.zeros(1, np.float32)), seed)
        got = _cache(B, ctx)
        tol = TOL["f32"] if shape.dtype == "f32" else TOL_BF16_OWN_PREFILL
        e = max(row_rel_err(got["glue_logits"][0], want.glue_logits), row_rel_err(got["logits"][0], want.logits))
        print(f"[scaled rotary] {scaling}, {name}, {pages} pages: {e:.2e}", flush=True)
        assert e < tol
        # (the plain frequencies are another model: the tolerance tells them apart)
        monkeypatch.undo()
        _, plain_trunk = O.prefill(om, prompt[0])
        plain, _, _ = O.glue_extend(om, plain_trunk, pending[0])
        assert row_rel_err(got["glue_logits"][0], plain) > 2 * tol
    finally:
        B.ssd_ctx_destroy(ctx)
        B.ssd_model_destroy(model)


def test_what_is_refused(B):
    model = B.ssd_model_create(F32, I.make_weights(F32, 1))
    try:
        for args in ((1, 3, 2, 128, B.SSD_CTX_PER_OPERATOR, 8), (1, 3, 2, 128, 0, 1)):
            with pytest.raises(B.SsdError) as e:
                B.ssd_ctx_create(model, *args)
            assert e.value.status == B.SSD_EINVAL
        for cfg in (B.rope_config(10000.0, 32), B.rope_config(10000.0, 64, layout="interleaved"), B.rope_config(0.5, 64),
                    B.rope_config(10000.0, 64, scaling="linear", factor=0.0)):
            with pytest.raises(B.SsdError) as e:
                B.ssd_model_set_rope(model, cfg)
            assert e.value.status == B.SSD_EINVAL
        with pytest.raises(B.SsdError):
            B._check(B.lib.ssd_model_set_rope(model, None))
    finally:
        B.ssd_model_destroy(model)
