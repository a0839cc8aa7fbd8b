"""Pins for the oracle's rotary positions and latent cache: the rotation against complex
products and its invariants, the tables against hand-derived values, the attention over
latent rows against the expanded heads' attention (keys and values projected first) and
against the ordinary paged oracle, the commit against a hand-built one."""
import numpy as np
import pytest

import oracle
from oracle import latent, status as st
from synth.batch import f32_to_bf16_bits


def _bf(x):
    return f32_to_bf16_bits(np.ascontiguousarray(x, np.float32)).reshape(np.shape(x))


@pytest.mark.parametrize("layout", [latent.HALF, latent.INTERLEAVED])
def test_rotation_is_a_complex_product(layout):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 3, 12))
    pos, f = np.array([0, 1, -7, 1000, 1 << 30]), 10.0 ** -np.arange(6)
    y = latent.rotate(x, pos, f, 1.5, layout)
    split = (lambda a: a[..., 0::2] + 1j * a[..., 1::2]) if layout else (lambda a: a[..., :6] + 1j * a[..., 6:])
    want = split(x) * 1.5 * np.exp(1j * (pos[:, None] * f))[:, None]
    assert np.abs(split(y) - want).max() < 1e-12
    assert np.array_equal(y[0], 1.5 * x[0])                         # position 0
    back = latent.rotate(y, pos, -f, 1 / 1.5, layout)               # negated frequencies turn back
    assert np.abs(back - x).max() < 1e-12
    # the gradient of sum(g y) with respect to x is the rotation of g by -f
    g = rng.standard_normal(x.shape)
    e = rng.standard_normal(x.shape)
    lhs = (g * latent.rotate(e, pos, f, 1.5, layout)).sum()
    assert abs(lhs - (latent.rotate(g, pos, -f, 1.5, layout) * e).sum()) < 1e-10


def test_scores_depend_on_distances_only():
    rng = np.random.default_rng(1)
    f, _ = latent.frequencies(64, 10000.0)
    q, k = rng.standard_normal((1, 64)), rng.standard_normal((1, 64))
    score = lambda p, c: float((latent.rotate(q, [p], f, 1.0, 0) * latent.rotate(k, [c], f, 1.0, 0)).sum())  # noqa: E731
    assert abs(score(10, 3) - score(1007, 1000)) < 1e-9


def test_frequencies_closed_forms():
    f, s = latent.frequencies(8, 10000.0)
    assert np.allclose(f, [1, 0.1, 0.01, 0.001]) and s == 1.0
    assert np.allclose(latent.frequencies(8, 10000.0, "linear", 4.0)[0], f / 4)
    # the first wave is kept, the last one stretched by the factor
    b, _ = latent.frequencies(8, 10000.0, "base", 16.0)
    assert np.isclose(b[0], 1.0) and np.isclose(b[-1], f[-1] / 16)
    # waves that turn more than high_turns times are kept, fewer than low_turns stretched
    m, _ = latent.frequencies(8, 10000.0, "smooth", 8.0, 2 * np.pi * 50, 1.0, 4.0)
    assert np.allclose(m, [1, 0.1, 0.01 / 8, 0.001 / 8])            # 50, 5, 0.5, 0.05 turns
    m, _ = latent.frequencies(8, 10000.0, "smooth", 8.0, 2 * np.pi * 25, 1.0, 4.0)
    assert np.isclose(m[1], 0.1 * (0.5 + 0.5 / 8))                  # 2.5 turns: half way
    y, s = latent.frequencies(8, 10000.0, "bands", 40.0, 2 * np.pi * 100, 1.0, 100.0)
    assert np.isclose(s, 0.1 * np.log(40) + 1)                      # 100 turns: pair 0, one turn: pair 2
    assert np.allclose(y, [1, 0.1 * (0.5 + 0.5 / 40), 0.01 / 40, 0.001 / 40])


def test_rows_of_the_projection():
    rng = np.random.default_rng(2)
    kv = _bf(rng.standard_normal((3, 576)))
    x = latent.bf16_to_f64(kv)
    assert np.array_equal(latent.latent_rows(kv, None, 0.0, None, None, 1.0, 0), x)
    one = _bf(np.ones(512))
    f, _ = latent.frequencies(64, 10000.0)
    y = latent.latent_rows(kv, one, 0.0, [0, 5, 9], f, 1.0, latent.HALF)
    assert np.allclose((y[:, :512] ** 2).mean(1), 1.0)              # unit mean square
    assert np.allclose(np.linalg.norm(y[:, 512:], axis=1), np.linalg.norm(x[:, 512:], axis=1))
    assert np.array_equal(y[0, 512:], x[0, 512:])
    zero = latent.latent_rows(np.zeros((1, 576), np.uint16), one, 1e-6, [3], f, 1.0, 0)
    assert np.all(zero == 0)


def _case(rng, hq, slots, plens, ps):
    R, cap = len(plens), sum(slots) + 2
    qo = np.zeros(R + 1, np.int32)
    qo[1:] = np.cumsum(slots)
    mask = np.zeros((cap, 1), np.uint32)
    for r in range(R):
        for j in range(slots[r]):
            up = mask[qo[r] + rng.integers(0, j), 0] if j else 0
            mask[qo[r] + j, 0] = up | np.uint32(1 << j)
    npg = [-(-p // ps) for p in plens]
    perm = rng.permutation(sum(npg) + 2)
    bt = np.full((R, max(npg)), -1, np.int32)
    at = 0
    for r in range(R):
        bt[r, :npg[r]] = perm[at:at + npg[r]]
        at += npg[r]
    return dict(q=_bf(rng.standard_normal((cap, hq, 576)) * 0.5), new=_bf(rng.standard_normal((cap, 576))),
                pages=_bf(rng.standard_normal((len(perm), ps, 576))), bt=bt, plen=np.array(plens, np.int32), qo=qo,
                mask=mask)


def test_attention_equals_expanded_heads():
    """Every head's own keys and values (projected from the latent rows, the rotated dims beside
    the keys), and softmax attention over them, against the latent rows with the projections
    absorbed into the query and left to the output.  Small whole numbers, so that the
    absorbed query is exact in bfloat16."""
    rng = np.random.default_rng(3)
    c = _case(rng, 2, [3, 1], [40, 0], 32)
    n, v = 16, 12  # the heads' own dims
    Wk, Wv = rng.integers(-2, 3, (2, n, 512)) / 8.0, rng.standard_normal((2, v, 512)) / 8
    qn = rng.integers(-1, 2, (c["q"].shape[0], 2, n)).astype(np.float64)
    qr = latent.bf16_to_f64(c["q"][..., 512:])
    for h in range(2):
        c["q"][:, h, :512] = _bf(qn[:, h] @ Wk[h])
    assert np.array_equal(latent.bf16_to_f64(c["q"][:, 1, :512]), qn[:, 1] @ Wk[1])
    ref = latent.tree_verify_attn_latent(c["q"], c["new"], c["pages"], c["bt"], c["plen"], c["qo"], c["mask"], 2, 0.07)
    assert ref["status"] == 0
    for r in range(2):
        P, q0, q1 = int(c["plen"][r]), int(c["qo"][r]), int(c["qo"][r + 1])
        C = np.concatenate([latent.cached_rows(c["pages"], c["bt"], r, P), latent.bf16_to_f64(c["new"][q0:q1])])
        for s in range(q0, q1):
            see = np.array([True] * P + [bool((int(c["mask"][s, 0]) >> j) & 1) for j in range(q1 - q0)])
            for h in range(2):
                keys, values = np.concatenate([C[:, :512] @ Wk[h].T, C[:, 512:]], 1), C[:, :512] @ Wv[h].T
                z = np.where(see, float(np.float32(0.07)) * (keys @ np.concatenate([qn[s, h], qr[s, h]])), -np.inf)
                p = np.exp(z - z.max())
                assert np.allclose((p / p.sum()) @ values, ref["out"][s, h] @ Wv[h].T, rtol=1e-9, atol=1e-9)


def test_attention_equals_the_paged_oracle():
    """Rows that are zero but in dims 0-127 are an ordinary cache of one KV head."""
    rng = np.random.default_rng(4)
    c = _case(rng, 4, [5, 0, 2], [70, 10, 0], 32)
    for k in ("q", "new", "pages"):
        c[k][..., 128:] = 0
    ref = latent.tree_verify_attn_latent(c["q"], c["new"], c["pages"], c["bt"], c["plen"], c["qo"], c["mask"], 4, 0.1)
    cut = lambda x: np.ascontiguousarray(x[..., :128])  # noqa: E731
    k, p = cut(c["new"])[:, None], cut(c["pages"])[:, :, None]
    out, lse, status = oracle.tree_verify_attn_paged(cut(c["q"]), k, k, p, p, c["bt"], c["plen"], 32, c["qo"], c["mask"],
                                                     4, 1, 0.1)
    assert status == ref["status"] == 0
    nq = int(c["qo"][-1])
    assert np.allclose(ref["out"][:nq, :, :128], out[:nq], atol=1e-12) and np.all(ref["out"][:nq, :, 128:] == 0)
    assert np.allclose(ref["lse"][:nq], lse[:nq], atol=1e-12)


def test_attention_rows_without_keys_and_bad_requests():
    rng = np.random.default_rng(5)
    c = _case(rng, 2, [2, 2, 1], [0, 40, 40], 32)
    c["mask"][0] = 0
    c["bt"][1, 1] = 99
    ref = latent.tree_verify_attn_latent(c["q"], c["new"], c["pages"], c["bt"], c["plen"], c["qo"], c["mask"], 2, 0.1)
    assert np.all(ref["out"][0] == 0) and np.all(np.isneginf(ref["lse"][0]))
    assert np.all(np.isnan(ref["lse"][2:4])) and ref["status"] == st.BAD_OFFSETS
    assert np.all(np.isfinite(ref["lse"][4]))


def test_commit_by_hand():
    pages = np.zeros((3, 32, 576), np.uint16)
    new = np.arange(6 * 576, dtype=np.uint16).reshape(6, 576)
    bt = np.array([[2, 0], [1, -1]], np.int32)
    got, ln, status = latent.commit_latent(np.array([0, 3, 6]), np.array([2, 1]), np.array([[1, 2], [4, -1]]), new,
                                           pages, bt, np.array([31, 31], np.int32))
    assert status == st.BAD_OFFSETS and list(ln) == [34, 31]        # the second lacks its second page
    assert np.array_equal(got[2, 31], new[0]) and np.array_equal(got[0, 0], new[1])
    assert np.array_equal(got[0, 1], new[2]) and not got[1].any()
