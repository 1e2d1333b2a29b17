"""The serving operators' refusals (no GPU needed: every argument is checked before anything is launched), and their float64 definitions
against direct statements of what they define."""
import ctypes as C

import numpy as np
import pytest

from oracle import serve_oracle as S


@pytest.fixture(scope="module")
def b():
    from paper_2603_03251_amd import binding
    return binding


def _rope(b, **over):
    r = b.rope_config(10000.0, 64)
    for k, v in over.items():
        setattr(r, k, v)
    return r


def _kv(b, **over):
    kv = b.ssd_paged_kv(4096, 8192, 64, 32 * 2 * 64, 4, 32, 8, 2, 64, b.SSD_BF16)
    for k, v in over.items():
        setattr(kv, k, v)
    return kv


def _refused(b, status, word):
    assert status == b.SSD_EINVAL
    assert word in b.lib.ssd_last_error().decode(), b.lib.ssd_last_error()


P = 4096      # a pointer that is never followed


@pytest.mark.parametrize("over,word", [
    (dict(rot_dim=0), "rot_dim"), (dict(rot_dim=63), "rot_dim"), (dict(rot_dim=66), "rot_dim"), (dict(layout=2), "layout"),
    (dict(scaling=4), "scaling"), (dict(scaling=-1), "scaling"), (dict(theta=1.0), "theta"), (dict(theta=float("nan")), "theta"),
    (dict(theta=float("inf")), "theta"), (dict(magnitude=0.0), "magnitude"), (dict(scaling=1, factor=0.0), "factor"),
    (dict(scaling=1, factor=float("nan")), "factor"), (dict(scaling=2, factor=2.0, low=1.0, high=1.0, original=100.0), "low < high"),
    (dict(scaling=2, factor=2.0, low=1.0, high=4.0, original=0.0), "original"), (dict(scaling=3, factor=2.0, low=0.0, high=4.0, original=9.0), "low"),
])
def test_rotary_settings_that_are_refused(b, over, word):
    _refused(b, b.lib.ssd_rope(_rope(b, **over), P, 256, b.SSD_F32, P, 3, 4, 64, P, 256, None), word)
    kv = _kv(b)
    _refused(b, b.lib.ssd_rope_append(_rope(b, **over), kv, P, 256, P, 128, P, 128, b.SSD_F32, P, None, 1, 1, 4, P, 256, None), word)


def test_rope_arguments_that_are_refused(b):
    ok = dict(rope=_rope(b), x=P, x_ld=256, dtype=b.SSD_F32, pos=P, rows=3, heads=4, dim=64, out=P, out_ld=256)

    def call(**over):
        return b.lib.ssd_rope(*{**ok, **over}.values(), None)

    for name in ("rope", "x", "pos", "out"):
        _refused(b, call(**{name: None}), "null")
    for over, word in [(dict(dim=80), "head_dim"), (dict(dim=32), "head_dim"), (dict(dtype=2), "dtype"), (dict(rows=-1), "rows"),
                       (dict(rows=(1 << 24) + 1), "rows"), (dict(heads=0), "heads"), (dict(rows=1 << 20, heads=300, x_ld=300 * 64, out_ld=300 * 64), "2^28"),
                       (dict(x_ld=255), "hold"), (dict(out_ld=255), "hold")]:
        _refused(b, call(**over), word)


CACHES = [(dict(d_k=None), "null"), (dict(d_v=None), "null"), (dict(d_table=None), "null"), (dict(dtype=7), "dtype"), (dict(head_dim=96), "head_dim"),
          (dict(n_kv_heads=0), "n_kv_heads"), (dict(page_size=4), "page_size"), (dict(page_size=48), "page_size"), (dict(page_size=2048), "page_size"),
          (dict(n_pages=0), "n_pages"), (dict(table_stride=0), "table_stride"), (dict(page_stride=32 * 2 * 64 - 8), "page_stride"),
          (dict(page_stride=32 * 2 * 64 + 4), "page_stride"), (dict(page_stride=1 << 62), "page_stride"), (dict(d_v=8200), "16 bytes")]


@pytest.mark.parametrize("over,word", CACHES)
def test_caches_that_are_refused(b, over, word):
    kv = _kv(b, **over)
    _refused(b, b.lib.ssd_rope_append(_rope(b), kv, P, 256, P, 128, P, 128, b.SSD_F32, P, None, 1, 1, 4, P, 256, None), word)
    _refused(b, b.lib.ssd_paged_attention(kv, P, 256, b.SSD_BF16, P, 1, 1, 4, 32, 0.125, None, P, 256, None, P, None), word)


def test_append_arguments_that_are_refused(b):
    ok = dict(rope=_rope(b), kv=_kv(b), q=P, q_ld=256, k=P, k_ld=128, v=P, v_ld=128, dtype=b.SSD_F32, pos=P, slots=None, B=1, T=1, heads=4,
              out=P, out_ld=256)

    def call(**over):
        return b.lib.ssd_rope_append(*{**ok, **over}.values(), None)

    for name in ("rope", "kv", "q", "k", "v", "pos", "out"):
        _refused(b, call(**{name: None}), "null")
    for over, word in [(dict(dtype=-1), "dtype"), (dict(B=-1), "B >= 0"), (dict(T=0), "T >= 1"), (dict(B=1 << 13, T=1 << 13), "2^24"), (dict(heads=0), "n_q_heads"),
                       (dict(q_ld=255), "hold"), (dict(k_ld=127), "hold"), (dict(v_ld=127), "hold"), (dict(out_ld=255), "hold")]:
        _refused(b, call(**over), word)


def test_attention_arguments_that_are_refused(b):
    ok = dict(kv=_kv(b), q=P, q_ld=256, dtype=b.SSD_BF16, vis=P, B=1, T=1, heads=4, most=256, scale=0.125, tail=None, out=P, out_ld=256, lse=None, ws=P)

    def call(**over):
        return b.lib.ssd_paged_attention(*{**ok, **over}.values(), None)

    for name in ("kv", "q", "vis", "out", "ws"):
        _refused(b, call(**{name: None}), "null")
    for over, word in [(dict(dtype=3), "dtype"), (dict(heads=3), "multiple"), (dict(heads=0), "multiple"), (dict(heads=2048, q_ld=1 << 18, out_ld=1 << 18), "1024"),
                       (dict(B=-1), "B in"), (dict(B=70000), "B in"), (dict(T=0), "T in"), (dict(B=65535, T=65535), "2^23"), (dict(T=65535, heads=64, q_ld=4096, out_ld=4096), "KV head"), (dict(most=-1), "max_visible"),
                       (dict(most=257), "block table"), (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"), (dict(q_ld=248), "hold"),
                       (dict(out_ld=248), "hold"), (dict(q=P + 8), "16 bytes"), (dict(out=P + 2), "16 bytes"), (dict(ws=P + 4), "16 bytes"),
                       (dict(q_ld=260), "16 bytes"), (dict(out_ld=258), "16 bytes"),
                       (dict(tail=b.ssd_tail_kv(None, P, 4, 4)), "tail"), (dict(tail=b.ssd_tail_kv(P, P, 4, 5)), "tail"),
                       (dict(tail=b.ssd_tail_kv(P, P, 257, 5)), "tail"), (dict(tail=b.ssd_tail_kv(P, P, 0, 0)), "tail"), (dict(tail=b.ssd_tail_kv(P, P, 4, -1)), "tail")]:
        _refused(b, call(**over), word)
    kv = _kv(b)
    assert b.ssd_paged_attention_workspace_bytes(kv, 1, 1, 4, 256) >= 4 * (64 + 2) * 4
    for bad in [(0, 1, 4, 256), (1, 0, 4, 256), (1, 1, 3, 256), (1, 1, 4, -1)]:
        assert b.ssd_paged_attention_workspace_bytes(kv, *bad) == 0


def test_verification_arguments_that_are_refused(b):
    ok = dict(p=P, p_ld=100, q=P, q_ld=100, spec=P, drafted=None, ua=P, ub=P, B=1, K=3, V=100, k=P, t=P, ws=P)

    def call(**over):
        return b.lib.ssd_verify_probs(*{**ok, **over}.values(), None)

    for name in ("p", "spec", "ua", "ub", "k", "t", "ws"):
        _refused(b, call(**{name: None}), "null")
    for over, word in [(dict(B=-1), "B"), (dict(B=65536), "B"), (dict(K=0), "K"), (dict(K=b.SSD_MAX_K + 1), "K"), (dict(V=1), "V"), (dict(p_ld=99), "hold"),
                       (dict(q_ld=99), "hold"), (dict(ws=P + 8), "16 bytes")]:
        _refused(b, call(**over), word)
    assert b.ssd_verify_probs_workspace_bytes(0, 100) == 0 and b.ssd_verify_probs_workspace_bytes(2, 0) == 0
    assert b.ssd_verify_probs_workspace_bytes(3, 1000) > b.ssd_verify_probs_workspace_bytes(1, 1000) > 0


def test_the_structures_have_the_headers_size(b):
    assert C.sizeof(b.ssd_rope_config) == 36 and C.sizeof(b.ssd_paged_kv) == 56 and C.sizeof(b.ssd_tail_kv) == 24


def test_frequencies_keep_fast_pairs_and_stretch_slow_ones():
    plain = S.rope_frequencies(500000.0, 128)
    assert plain[0] == 1.0 and np.all(np.diff(plain) < 0)
    for scaling in ("bands", "ramp"):
        f = S.rope_frequencies(500000.0, 128, scaling, 8.0, 1.0, 4.0 if scaling == "bands" else 32.0, 8192.0)
        ratio = f / plain
        assert ratio[0] == 1.0 and abs(ratio[-1] - 1 / 8) < 1e-15 and np.all(np.diff(ratio) <= 1e-15)
        assert np.any((ratio > 0.13) & (ratio < 0.99))
    assert np.allclose(S.rope_frequencies(10000.0, 64, "linear", 4.0), S.rope_frequencies(10000.0, 64) / 4.0, rtol=1e-15)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotations_keep_products_of_equal_distance(layout):
    g = np.random.default_rng(1)
    q, k = g.standard_normal((1, 64)), g.standard_normal((1, 64))
    f = S.rope_frequencies(10000.0, 32)
    dot = lambda m, n: float((S.rotate(q, np.array(m), f, layout)[0] * S.rotate(k, np.array(n), f, layout)[0]).sum())
    assert abs(dot(17, 5) - dot(1017, 1005)) < 1e-10 and abs(dot(17, 5) - dot(17, 6)) > 1e-6


def test_verification_emits_the_targets_distribution():
    """The first emitted token of a round is distributed as the target's first row, whatever the draft's distribution."""
    g = np.random.default_rng(7)
    V, n = 6, 20000
    p, q = g.dirichlet(np.ones(V), 2), g.dirichlet(np.ones(V), 1)
    p[0, 2] = 0.0
    p[0] /= p[0].sum()
    seen = np.zeros(V)
    for _ in range(n):
        s = g.choice(V, p=q[0])
        k, t = S.verify_probs(p, q, np.array([s]), g.random(1), g.random())
        seen[s if k else t] += 1
    # five standard deviations of a count of n draws
    assert np.all(np.abs(seen / n - p[0]) <= 5 * np.sqrt(p[0] * (1 - p[0]) / n) + 1e-12)
