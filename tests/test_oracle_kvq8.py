"""Pins for the oracle's 8-bit cache and block tables: the number formats against every byte
and torch's conversions, the scales and appends against hand-derived values and
invariants, attention against the bf16 oracle on exactly representable values, the
tables against conservation of pages."""
import numpy as np
import pytest
import torch

import oracle
from oracle import kvq8, status as st
from synth.batch import f32_to_bf16_bits

TORCH = {kvq8.E4M3: torch.float8_e4m3fn, kvq8.E5M2: torch.float8_e5m2}
FMTS = (kvq8.E4M3, kvq8.E5M2)


def _bf(x):
    return f32_to_bf16_bits(np.ascontiguousarray(x, np.float32)).reshape(np.shape(x))


@pytest.mark.parametrize("fmt", FMTS)
def test_formats_match_torch(fmt):
    b = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(b).view(TORCH[fmt]).to(torch.float64).numpy()
    got = kvq8.decode8(b, fmt)
    assert np.array_equal(got, want, equal_nan=True)
    fin = b[np.isfinite(got)]
    assert np.array_equal(kvq8.encode8(kvq8.decode8(fin, fmt), fmt), fin)
    # between neighbours: below, at and above each midpoint
    mag = np.sort(np.unique(np.abs(kvq8.decode8(fin, fmt))))
    mid = 0.5 * (mag[1:] + mag[:-1])
    x = np.concatenate([mid, mid * (1 - 1e-6), mid * (1 + 1e-6)])
    x = np.concatenate([x, -x]).astype(np.float32)
    want = torch.from_numpy(x).to(TORCH[fmt]).view(torch.uint8).numpy()
    assert np.array_equal(kvq8.encode8(x.astype(np.float64), fmt), want)
    top = kvq8.FORMATS[fmt][2]
    assert np.array_equal(kvq8.decode8(kvq8.encode8(np.array([1e30, -np.inf]), fmt), fmt), [top, -top])
    assert np.isnan(kvq8.decode8(kvq8.encode8(np.array([np.nan]), fmt), fmt))[0]


def test_scale_closed_forms():
    one = lambda *v: np.array(v, np.float64)  # noqa: E731
    assert kvq8.need_scale(one(448.0), kvq8.E4M3) == 1.0
    assert kvq8.need_scale(one(450.0), kvq8.E4M3) == 2.0
    assert kvq8.need_scale(one(-3.5, 1.0), kvq8.E4M3) == 2.0 ** -7
    assert kvq8.need_scale(one(57344.0), kvq8.E5M2) == 1.0
    assert kvq8.need_scale(one(0.0), kvq8.E4M3) == 2.0 ** -60
    assert kvq8.need_scale(one(np.inf, np.nan, 448.0), kvq8.E4M3) == 1.0
    assert kvq8.need_scale(one(3e38), kvq8.E4M3) == 2.0 ** 60


def test_append_grows_the_scale_and_keeps_values():
    """1.0 at scale 2^-8 (byte 256 -> 448 is the largest), then 400: the scale becomes 1 and the
    first row keeps its value; a value that becomes subnormal is rounded."""
    k = np.zeros((1, 1, 32, 128), np.uint8)
    s = np.full((1, 1, 1), 99.0, np.float32)           # whatever the scale held
    x = np.zeros((1, 1, 128))
    x[0, 0, :3] = 1.0, -1.75, 2.0 ** -14               # 2^-14 = 2^-6 at scale 2^-8
    kvq8.append_rows(k, s, kvq8.E4M3, 0, 0, x)
    assert s[0, 0, 0] == 2.0 ** -8
    assert np.array_equal(kvq8.decode8(k[0, 0, 0, :3], kvq8.E4M3) * 2.0 ** -8, x[0, 0, :3])
    y = np.full((2, 1, 128), 400.0)
    kvq8.append_rows(k, s, kvq8.E4M3, 0, 1, y)
    assert s[0, 0, 0] == 1.0
    assert np.array_equal(kvq8.decode8(k[0, 0, 0, :3], kvq8.E4M3), [1.0, -1.75, 0.0])
    assert np.all(kvq8.decode8(k[0, 0, 1:3], kvq8.E4M3) == 384.0)  # a midpoint: the even one


@pytest.mark.parametrize("fmt", FMTS)
def test_store_in_pieces_keeps_the_rounding_bound(fmt):
    """Every stored value is within the rounding of its format of what was given (one half step
    for each of the at most two roundings that a value below the normal range sees)."""
    rng = np.random.default_rng(fmt)
    x = _bf(rng.standard_normal((70, 2, 128)) * np.exp2(rng.integers(-3, 4, (70, 2, 1))))
    pages, ps = 3, 64
    cache = [np.full((pages, 2, ps, 128), 0x7F, np.uint8) for _ in range(2)]
    cache += [np.full((pages, 2, ps // 32), np.nan, np.float32) for _ in range(2)]
    cuts = [0, 1, 5, 30, 33, 40, 70]
    slots = np.array([64 + p if p < 64 else p - 64 for p in range(70)], np.int64)  # page 1, then 0
    for a, b in zip(cuts, cuts[1:]):
        *cache, status = kvq8.store_kv(x[a:b], x[a:b], slots[a:b], fmt, *cache)
        assert status == 0
    bias, man, _ = kvq8.FORMATS[fmt]
    v = kvq8.bf16_to_f64(x)
    for p in range(70):
        pg, o = int(slots[p]) // ps, int(slots[p]) % ps
        for h in range(2):
            s = float(cache[2][pg, h, o // 32])
            got = kvq8.decode8(cache[0][pg, h, o], fmt) * s
            step = np.maximum(np.abs(v[p, h]) * 2.0 ** -(man + 1), 2 * s * 2.0 ** (-bias - man))
            assert np.all(np.abs(got - v[p, h]) <= step)
    # the rows behind are as they were
    assert np.all(cache[0][0, :, 6:] == 0x7F) and np.all(cache[0][2] == 0x7F)
    assert np.isnan(cache[2][2]).all()


def test_store_leaves_out_bad_slots():
    x = _bf(np.ones((4, 1, 128)))
    cache = [np.zeros((1, 1, 32, 128), np.uint8) for _ in range(2)]
    cache += [np.ones((1, 1, 1), np.float32) for _ in range(2)]
    *got, status = kvq8.store_kv(x, x, [-1, 0, 32, 1], kvq8.E4M3, *cache)
    assert status == st.BAD_OFFSETS
    assert np.count_nonzero(got[0].any(-1)) == 2


def test_attention_on_representable_values_is_the_bf16_oracle():
    rng = np.random.default_rng(5)
    hq, hkv, ps, plen = 4, 2, 32, np.array([40, 0, 7], np.int32)
    small = lambda *s: _bf(rng.integers(-7, 8, s).astype(np.float32) / 4)  # noqa: E731
    qo = np.array([0, 3, 4, 6], np.int32)
    mask = np.array([1, 3, 5, 1, 0, 2], np.uint32)[:, None]  # a row that sees only the prefix
    q, kn, vn = small(6, hq, 128), small(6, hkv, 128), small(6, hkv, 128)
    bt = np.array([[2, 0], [-1, -1], [1, -1]], np.int32)
    kb, vb = small(3, ps, hkv, 128), small(3, ps, hkv, 128)  # token-major, as the bf16 cache
    enc = lambda b: kvq8.encode8(kvq8.bf16_to_f64(b) / 4.0, kvq8.E4M3).transpose(0, 2, 1, 3)  # noqa: E731
    sc = np.full((3, hkv, 1), 4.0, np.float32)
    got = kvq8.tree_verify_attn_paged_q8(q, kn, vn, kvq8.E4M3, enc(kb), enc(vb), sc, sc, bt, plen, qo,
                                         mask, hq, hkv, 0.3)
    want, lse, status = oracle.tree_verify_attn_paged(q, kn, vn, kb, vb, bt, plen, ps, qo, mask, hq,
                                                      hkv, 0.3)
    assert got["status"] == status == 0
    assert np.allclose(got["out"], want, rtol=0, atol=1e-12)
    assert np.allclose(got["lse"], lse, rtol=0, atol=1e-12)
    bt[0, 1] = 3                                             # a page that does not exist
    got = kvq8.tree_verify_attn_paged_q8(q, kn, vn, kvq8.E4M3, enc(kb), enc(vb), sc, sc, bt, plen, qo,
                                         mask, hq, hkv, 0.3)
    assert got["status"] == st.BAD_OFFSETS and np.isnan(got["out"][:3]).all()
    assert np.allclose(got["out"][3:], want[3:], rtol=0, atol=1e-12)


def test_commit_is_a_store_of_the_accepted_rows():
    rng = np.random.default_rng(2)
    kn, vn = (_bf(rng.standard_normal((5, 2, 128))) for _ in range(2))
    cache = [np.zeros((4, 2, 32, 128), np.uint8) for _ in range(2)]
    cache += [np.ones((4, 2, 1), np.float32) for _ in range(2)]
    qo, al = np.array([0, 3, 3, 5], np.int32), np.array([2, 0, 1], np.int32)
    acc = np.array([[1, 2], [-1, -1], [4, -1]], np.int32)
    bt, plen = np.array([[3, 0], [1, -1], [-1, -1]], np.int32), np.array([30, 5, 0], np.int32)
    *got, new_len, status = kvq8.commit_kv_q8(qo, al, acc, kn, vn, kvq8.E5M2, *cache, bt, plen)
    assert status == st.BAD_OFFSETS and new_len.tolist() == [33, 5, 0]  # request 2 has no page
    *want, _ = kvq8.store_kv(kn[:3], vn[:3], [3 * 32 + 30, 3 * 32 + 31, 0], kvq8.E5M2, *cache)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)


def test_tables_hand_derived():
    """Pages of 4 tokens: request 0 ends (gives 5, 6), request 1 grows by one page (takes 6), 2
    keeps its page, 3 wants three (5 and the stack's 9, 8), 4 finds nothing left."""
    bt = np.array([[5, 6, -1], [7, -1, -1], [2, -1, -1], [-1, -1, -1], [-1, -1, -1]], np.int32)
    got = kvq8.build_block_tables([0, 5, 4, 12, 1], 4, bt, [2, 1, 1, 0, 0], np.array([8, 9, -1, -1]), 2,
                                  [0, 0, 1, 1, 3, 4], [8, 4, 3, 0, 0], 6)
    assert got["num_held"].tolist() == [0, 2, 1, 3, 0] and got["num_free"] == 0
    assert got["block_table"][1].tolist() == [7, 6, -1]
    assert got["block_table"][3].tolist() == [5, 9, 8]
    assert got["slot_map"].tolist() == [6 * 4, 5 * 4, 5 * 4 + 1, -1, -1, -1]
    assert got["status"] == st.NO_PAGES


@pytest.mark.parametrize("seed", range(8))
def test_tables_conserve_pages(seed):
    rng = np.random.default_rng(seed)
    R, most, ps = 9, 6, 8
    held = rng.integers(0, most + 1, R)
    total = int(held.sum()) + 7
    perm = rng.permutation(total)
    bt = np.full((R, most), -1, np.int32)
    at = 0
    for r in range(R):
        bt[r, :held[r]] = perm[at:at + held[r]]
        at += held[r]
    stack = np.full(total, -1, np.int32)
    stack[:7] = perm[at:]
    want = rng.integers(0, most * ps + 1, R)
    got = kvq8.build_block_tables(want, ps, bt, held, stack, 7)
    pages = [int(p) for r in range(R) for p in got["block_table"][r, :got["num_held"][r]]]
    pages += got["free_pages"][:got["num_free"]].tolist()
    assert sorted(pages) == list(range(total))
    need = -(-want // ps)
    for r in range(R):
        assert got["num_held"][r] == need[r] or (got["num_held"][r] == held[r] < need[r])
        keep = min(held[r], got["num_held"][r])
        assert np.array_equal(got["block_table"][r, :keep], bt[r, :keep])
