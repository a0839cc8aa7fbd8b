"""GPU parity of the 8-bit paged cache's writers, of the block tables and of the attention
over the cache, against the oracle: bytes, scales, tables and slots exactly, attention
within the roundings that the call documents."""
import numpy as np
import pytest

from oracle import kvq8, status as st
from synth.batch import f32_to_bf16_bits
from tests import gpu_common as gc

pytestmark = pytest.mark.gpu
FMTS = (kvq8.E4M3, kvq8.E5M2)


@pytest.fixture(autouse=True)
def _need_gpu():
    gc.require_gpu()


def _log(msg):
    print(msg, flush=True)


def _dev(a):
    import torch
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        a = a.view(np.int16)
    if a.dtype == np.uint32:
        a = a.view(np.int32)
    return torch.from_numpy(a).to("cuda:0")


def _bf(x):
    return f32_to_bf16_bits(np.ascontiguousarray(x, np.float32)).reshape(np.shape(x))


def _zeros(*s):
    import torch
    return torch.zeros(s, dtype=torch.int32, device="cuda:0")


def _values(rng, *shape):
    """bf16 values whose magnitudes differ from row to row, zeros among them."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-4, 5, shape[:-1] + (1,)))
    x[rng.random(shape[:-1]) < 0.05] = 0.0
    return _bf(x)


def _empty_cache(rng, pages, hkv, ps):
    """A cache of arbitrary bytes and scales: what no call has written."""
    c = [rng.integers(0, 256, (pages, hkv, ps, 128)).astype(np.uint8) for _ in range(2)]
    return c + [np.exp2(rng.integers(-9, 9, (pages, hkv, ps // 32))).astype(np.float32) for _ in range(2)]


def _same_bytes(got, want, fmt, what):
    """Equal bytes; NaN of either sign and payload is the same."""
    bad = got != want
    if bad.any():
        nan = np.isnan(kvq8.decode8(got[bad], fmt)) & np.isnan(kvq8.decode8(want[bad], fmt))
        assert nan.all(), (what, int((~nan).sum()), np.argwhere(bad)[0])


def _store(k, v, slots, fmt, cache, ps, status=None, stream=None):
    import paper_2604_09603_amd as pkg
    pkg.echo_store_kv_q8(k, v, slots, len(slots), k.shape[1], 128, fmt, *cache, ps, status=status,
                         stream=stream)


def _slots_of(lens, starts, ps, rng, spare=2):
    """Slots of rows [start, start + len) of each request over shuffled pages; the pool's
    pages, and the table."""
    npg = [-(-(s + n) // ps) for s, n in zip(starts, lens)]
    perm = rng.permutation(sum(npg) + spare)
    bt = np.full((len(lens), max(max(npg), 1)), -1, np.int32)
    at, slots = 0, []
    for r, (n, s) in enumerate(zip(lens, starts)):
        bt[r, :npg[r]] = perm[at:at + npg[r]]
        at += npg[r]
        p = np.arange(s, s + n)
        slots.append(bt[r, p // ps].astype(np.int64) * ps + p % ps)
    return np.concatenate(slots), len(perm), bt


# ---- store ----------------------------------------------------------------

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hkv,ps,lens,starts", [
    (1, 32, [1], [0]), (2, 32, [1, 1, 1], [0, 31, 17]), (3, 64, [31, 32, 33, 64], [0, 0, 0, 0]),
    (8, 64, [5, 100, 1, 40], [30, 61, 95, 32]), (5, 256, [300, 1, 2], [250, 1, 63]),
    (4, 128, [1] * 70, list(range(70)))])
def test_store_matches_oracle(fmt, hkv, ps, lens, starts):
    rng = np.random.default_rng(len(lens) * 100 + hkv)
    slots, pages, _ = _slots_of(lens, starts, ps, rng)
    T = len(slots)
    k, v = _values(rng, T, hkv, 128), _values(rng, T, hkv, 128)
    cache = _empty_cache(rng, pages, hkv, ps)
    dev = [_dev(a) for a in cache]
    status = _zeros(1)
    _log(f"[store] fmt={fmt} hkv={hkv} page={ps} T={T}")
    _store(_dev(k), _dev(v), _dev(slots), fmt, dev, ps, status)
    *want, wst = kvq8.store_kv(k, v, slots, fmt, *cache)
    assert int(status.item()) == wst == 0
    for i in range(2):
        _same_bytes(dev[i].cpu().numpy(), want[i], fmt, f"tensor {i}")
        assert np.array_equal(dev[2 + i].cpu().numpy(), want[2 + i])


@pytest.mark.parametrize("fmt", FMTS)
def test_store_special_values(fmt):
    """NaN and infinities don't enter a scale; zero blocks, the smallest and the largest
    values, the border of a scale."""
    rng = np.random.default_rng(0)
    T, hkv, ps = 160, 2, 32
    x = _values(rng, T, hkv, 128)
    x[3, 0, 5], x[4, 0, 6], x[5, 1, 7], x[6, 1, 8] = 0x7FC0, 0xFF80, 0x7F80, 0xFFFF
    x[32:64] = 0
    x[64:96] = _bf(rng.standard_normal((32, hkv, 128)) * 1e-38)
    x[96:128] = _bf(rng.standard_normal((32, hkv, 128)) * 1e38)
    x[128:160] = _bf(np.clip(rng.standard_normal((32, hkv, 128)), -1, 1))
    x[130, 0, 0], x[131, 1, 1] = _bf([448.0 if fmt == kvq8.E4M3 else 57344.0])[0], 0x43E1  # 450
    cache = _empty_cache(rng, 5, hkv, ps)
    dev = [_dev(a) for a in cache]
    slots = np.arange(T, dtype=np.int64)
    _log(f"[store] special values fmt={fmt}")
    _store(_dev(x), _dev(x[::-1].copy()), _dev(slots), fmt, dev, ps)
    *want, _ = kvq8.store_kv(x, x[::-1], slots, fmt, *cache)
    for i in range(2):
        assert np.array_equal(dev[2 + i].cpu().numpy(), want[2 + i])
        _same_bytes(dev[i].cpu().numpy(), want[i], fmt, f"tensor {i}")


@pytest.mark.parametrize("fmt", FMTS)
def test_store_appends_in_pieces(fmt):
    """Uneven pieces into the same blocks, scales that grow and others that don't."""
    rng = np.random.default_rng(7 + fmt)
    hkv, ps, T = 3, 64, 200
    slots, pages, _ = _slots_of([T], [0], ps, rng)
    k, v = _values(rng, T, hkv, 128), _values(rng, T, hkv, 128)
    cache = _empty_cache(rng, pages, hkv, ps)
    dev = [_dev(a) for a in cache]
    want = cache
    cuts = np.unique(np.concatenate([[0, T], rng.integers(1, T, 40)]))
    for a, b in zip(cuts, cuts[1:]):
        _log(f"[store] fmt={fmt} rows {a}..{b}")
        _store(_dev(k[a:b]), _dev(v[a:b]), _dev(slots[a:b]), fmt, dev, ps)
        *want, _ = kvq8.store_kv(k[a:b], v[a:b], slots[a:b], fmt, *want)
    for i in range(2):
        assert np.array_equal(dev[2 + i].cpu().numpy(), want[2 + i])
        _same_bytes(dev[i].cpu().numpy(), want[i], fmt, f"tensor {i}")


@pytest.mark.parametrize("old", [1.3, 0.7])
def test_store_into_a_block_with_another_scale(old):
    """A part-filled block whose scale is no power of two keeps it where the new rows need less
    (they are divided by it), and takes a power of two where they need more.  Every value is within
    half a step of the exact one, and a half step of fp32 (2^-24 of it) where that decides."""
    rng = np.random.default_rng(3)
    ps, fmt = 32, kvq8.E4M3
    cache = _empty_cache(rng, 1, 2, ps)
    for i in range(2):
        cache[i] = kvq8.encode8(rng.standard_normal(cache[i].shape) * 50, fmt)
        cache[2 + i][:] = old
    x = _bf(rng.standard_normal((9, 2, 128)) * 100)
    x[:, 1] = _bf(rng.standard_normal((9, 128)) * 1000)  # head 1: the scale grows
    dev = [_dev(a) for a in cache]
    _store(_dev(x), _dev(x), _dev(np.arange(11, 20, dtype=np.int64)), fmt, dev, ps)
    got = dev[0].cpu().numpy()
    s = dev[2].cpu().numpy()[0, :, 0]
    for h in range(2):
        need = kvq8.need_scale(kvq8.bf16_to_f64(x[:, h]), fmt)
        assert s[h] == max(np.float32(old), np.float32(need))
        for exact, at in ((kvq8.decode8(cache[0][0, h, :11], fmt) * (float(np.float32(old)) / s[h]),
                           got[0, h, :11]),
                          (kvq8.bf16_to_f64(x[:, h]) / float(s[h]), got[0, h, 11:20])):
            val = kvq8.decode8(at, fmt)
            assert np.all(np.abs(val - exact) <= np.maximum(np.abs(exact) * 2.0 ** -4, 2.0 ** -10) *
                          (1 + 2.0 ** -20))
        assert np.array_equal(got[0, h, 20:], cache[0][0, h, 20:])


def test_store_padding_bad_slots_and_strides():
    """Negative slots are padding, slots past the pool are reported, rows of one projection's
    output are strided."""
    rng = np.random.default_rng(11)
    hkv, ps, T = 2, 32, 90
    cache = _empty_cache(rng, 4, hkv, ps)
    dev = [_dev(a) for a in cache]
    kv = _values(rng, T, 3, hkv, 128)
    slots = np.arange(T, dtype=np.int64)
    slots[5:9] = -1
    slots[40] = 4 * ps
    slots[41] = np.iinfo(np.int64).max
    slots[80:] = np.iinfo(np.int64).min
    t = _dev(kv)
    status = _zeros(1)
    _log("[store] padding, bad slots, strides")
    _store(t[:, 0], t[:, 2], _dev(slots), kvq8.E4M3, dev, ps, status)
    *want, wst = kvq8.store_kv(kv[:, 0], kv[:, 2], slots, kvq8.E4M3, *cache)
    assert int(status.item()) == wst == st.BAD_OFFSETS
    # the gaps leave two runs each in the pages 0 and 1, which are unspecified then
    for i in range(2):
        _same_bytes(dev[i].cpu().numpy()[2:], want[i][2:], kvq8.E4M3, f"tensor {i}")
        assert np.array_equal(dev[2 + i].cpu().numpy()[2:], want[2 + i][2:])
    # padding and bad slots between runs of different blocks
    dev = [_dev(a) for a in cache]
    slots = np.concatenate([np.arange(96, 101), [-1] * 4, np.arange(0, 31), [4 * ps, 1 << 40],
                            np.arange(32, 64), [-(1 << 40)], np.arange(64, 70), [-1] * 9])
    assert len(slots) == T
    _store(t[:, 0], t[:, 2], _dev(slots), kvq8.E4M3, dev, ps, status)
    *want, _ = kvq8.store_kv(kv[:, 0], kv[:, 2], slots, kvq8.E4M3, *cache)
    for i in range(2):
        _same_bytes(dev[i].cpu().numpy(), want[i], kvq8.E4M3, f"tensor {i}")
        assert np.array_equal(dev[2 + i].cpu().numpy(), want[2 + i])


@pytest.mark.parametrize("T", [2047, 2048, 2049, 5000])
def test_store_long_prompts(T):
    """Around the number of rows up to which every row has waves of its own: prompts, and
    single tokens between them, against a store row block by row block."""
    rng = np.random.default_rng(T)
    hkv, ps = 2, 64
    lens = [1, 1, 700, 1, 1, 33, 600]
    lens.append(T - sum(lens))
    starts = [3, 40, 17, 63, 0, 5, 0, 31]
    slots, pages, _ = _slots_of(lens, starts, ps, rng)
    k, v = _values(rng, T, hkv, 128), _values(rng, T, hkv, 128)
    cache = _empty_cache(rng, pages, hkv, ps)
    dev = [_dev(a) for a in cache]
    _log(f"[store] T={T}")
    _store(_dev(k), _dev(v), _dev(slots), kvq8.E4M3, dev, ps)
    *want, _ = kvq8.store_kv(k, v, slots, kvq8.E4M3, *cache)
    for i in range(2):
        _same_bytes(dev[i].cpu().numpy(), want[i], kvq8.E4M3, f"tensor {i}")
        assert np.array_equal(dev[2 + i].cpu().numpy(), want[2 + i])


@pytest.mark.parametrize("T", [256, 257, 600, 1025, 2050, 4097, 9000])
def test_store_rows_per_wave(T):
    """Every number of rows that a wave takes (eight heads: 1 at 256 rows, 32 from 4097 on), with
    runs that begin and end at any row of its chunk."""
    rng = np.random.default_rng(T)
    hkv, ps = 8, 64
    lens, starts = [], []
    while sum(lens) < T:
        n = int(rng.choice([1, 1, 2, 7, 31, 33, 64, 200]))
        lens.append(min(n, T - sum(lens)))
        starts.append(int(rng.integers(0, 70)))
    slots, pages, _ = _slots_of(lens, starts, ps, rng)
    k, v = _values(rng, T, hkv, 128), _values(rng, T, hkv, 128)
    cache = _empty_cache(rng, pages, hkv, ps)
    dev = [_dev(a) for a in cache]
    _log(f"[store] rows per wave, T={T}")
    _store(_dev(k), _dev(v), _dev(slots), kvq8.E5M2, dev, ps)
    *want, _ = kvq8.store_kv(k, v, slots, kvq8.E5M2, *cache)
    for i in range(2):
        _same_bytes(dev[i].cpu().numpy(), want[i], kvq8.E5M2, f"tensor {i}")
        assert np.array_equal(dev[2 + i].cpu().numpy(), want[2 + i])


# ---- commit ---------------------------------------------------------------

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hkv,ps,alias", [(1, 32, False), (4, 64, True), (9, 256, False)])
def test_commit_matches_oracle(fmt, hkv, ps, alias):
    """Paths of 0..16 accepted slots over block and page borders; a request without slots, a
    missing page, a bad slot, a bad length."""
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(hkv)
    R, depth = 14, 16
    plen = np.array([0, 31, 32, 63, 5, 20, 16, 100, 33, 47, 7, 60, 1, 15], np.int32)
    acc_len = np.array([0, 16, 3, 2, 16, 12, 15, 1, 4, 0, 5, 6, 16, 16], np.int32)
    qo = np.zeros(R + 1, np.int32)
    nslots = np.where(np.arange(R) == 9, 0, acc_len + 1 + rng.integers(0, 4, R))
    qo[1:] = np.cumsum(nslots)
    acc = np.full((R, depth), -1, np.int32)
    for r in range(R):
        if nslots[r]:
            acc[r, :acc_len[r]] = qo[r] + np.sort(rng.choice(np.arange(1, nslots[r]), acc_len[r], False))
    _, pages, bt = _slots_of([depth + 1] * R, plen.tolist(), ps, rng)
    bt[4, :] = -1                       # no pages
    acc[8, 1] = int(qo[-1])             # a slot that does not exist
    acc_len[10] = 17                    # more than max_depth
    cap = int(qo[-1])
    kn, vn = _values(rng, cap, hkv, 128), _values(rng, cap, hkv, 128)
    cache = _empty_cache(rng, pages, hkv, ps)
    dev = [_dev(a) for a in cache]
    status, pl = _zeros(1), _dev(plen)
    new = pl if alias else _zeros(R)
    _log(f"[commit] fmt={fmt} hkv={hkv} page={ps}")
    pkg.echo_commit_kv_q8(_dev(qo), _dev(acc_len), _dev(acc), depth, _dev(kn), _dev(vn), R, cap, hkv, 128,
                          fmt, *dev, ps, _dev(bt), pl, new, status=status)
    want_len, want_acc = acc_len.copy(), acc.copy()
    want_acc[10, :] = cap               # (the oracle refuses it by its slots)
    want_len[10] = 1
    *want, new_len, wst = kvq8.commit_kv_q8(qo, want_len, want_acc, kn, vn, fmt, *cache, bt, plen)
    assert int(status.item()) == wst == st.BAD_OFFSETS
    assert np.array_equal(new.cpu().numpy(), new_len)
    assert new_len[4] == plen[4] and new_len[8] == plen[8] and new_len[9] == plen[9]
    for i in range(2):
        _same_bytes(dev[i].cpu().numpy(), want[i], fmt, f"tensor {i}")
        assert np.array_equal(dev[2 + i].cpu().numpy(), want[2 + i])


# ---- block tables -----------------------------------------------------------

def _tables_case(rng, R, most, ps, free, rows, refuse=False):
    held = rng.integers(0, most + 1, R).astype(np.int32)
    total = int(held.sum()) + free
    perm = rng.permutation(total).astype(np.int32)
    bt = np.full((R, most), -1, np.int32)
    at = 0
    for r in range(R):
        bt[r, :held[r]] = perm[at:at + held[r]]
        at += int(held[r])
    stack = np.full(total + 3, -5, np.int32)
    stack[:free] = perm[at:]
    want = rng.integers(0, most * ps + 1, R).astype(np.int32)
    want[rng.random(R) < 0.3] = 0
    if refuse:
        want[R // 3], held[R // 2], held[R - 1] = -4, most + 1, -1
        want[0] = most * ps + 1
    n = rng.multinomial(rows, np.ones(R) / R)
    ro = np.zeros(R + 1, np.int32)
    ro[1:] = np.cumsum(n)
    start = np.maximum(0, want - n).astype(np.int32)
    return dict(want=want, held=held, bt=bt, stack=stack, free=free, ro=ro, start=start)


def _run_tables(c, R, ps, max_rows, alias, slot_map=True):
    import torch
    import paper_2604_09603_amd as pkg
    bt, stack, held, free, status = (_dev(c["bt"]), _dev(c["stack"]), _dev(c["held"]),
                                     _dev(np.array([c["free"]], np.int32)), _zeros(1))
    held_out, free_out = (held, free) if alias else (_zeros(R), _zeros(1))
    sm = torch.full((max_rows,), -77, dtype=torch.int64, device="cuda:0") if slot_map else None
    pkg.echo_build_block_tables(_dev(c["want"]), R, ps, bt, held, held_out, stack, free, free_out,
                                row_offsets=_dev(c["ro"]) if slot_map else None,
                                row_start=_dev(c["start"]) if slot_map else None, slot_map=sm, status=status)
    return dict(block_table=bt.cpu().numpy(), num_held=held_out.cpu().numpy(), free_pages=stack.cpu().numpy(),
                num_free=int(free_out.item()), slot_map=None if sm is None else sm.cpu().numpy(),
                status=int(status.item()))


def _same_tables(got, want):
    for n in ("num_held", "num_free", "free_pages", "status"):
        assert np.array_equal(got[n], want[n]), n
    assert np.array_equal(got["block_table"], want["block_table"])
    if got["slot_map"] is not None:
        assert np.array_equal(got["slot_map"], want["slot_map"])


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("R,most,ps,free,rows,pad", [
    (1, 1, 1, 0, 1, 0), (1, 5, 16, 9, 3, 1), (7, 6, 32, 4, 50, 9), (128, 9, 64, 300, 4000, 96),
    (128, 9, 64, 300, 4000, 97), (300, 4, 32, 900, 9000, 5), (1024, 3, 64, 10, 2000, 0),
    (1025, 2, 8, 1500, 100, 3), (4095, 2, 16, 3000, 12345, 11)])
def test_tables_match_oracle(R, most, ps, free, rows, pad, alias):
    rng = np.random.default_rng(R + rows)
    c = _tables_case(rng, R, most, ps, free, rows)
    _log(f"[tables] R={R} most={most} page={ps} free={free} rows={rows}+{pad}")
    got = _run_tables(c, R, ps, rows + pad, alias)
    want = kvq8.build_block_tables(c["want"], ps, c["bt"], c["held"], c["stack"], c["free"], c["ro"],
                                   c["start"], rows + pad)
    _same_tables(got, want)


@pytest.mark.parametrize("R,most,ps,free,rows,pad", [
    (128, 9, 64, 300, 2000, 48), (128, 9, 64, 300, 2000, 49), (4095, 2, 16, 3000, 2000, 11),
    (4095, 2, 16, 3000, 0, 1)])
def test_tables_and_slots_in_one_launch_or_two(R, most, ps, free, rows, pad):
    """The longest slot map that the tables' launch writes and the shortest of a launch of its own;
    the largest batch in one launch."""
    rng = np.random.default_rng(R + rows + pad)
    c = _tables_case(rng, R, most, ps, free, rows)
    _log(f"[tables] R={R} rows={rows}+{pad}")
    got = _run_tables(c, R, ps, rows + pad, False)
    want = kvq8.build_block_tables(c["want"], ps, c["bt"], c["held"], c["stack"], c["free"], c["ro"],
                                   c["start"], rows + pad)
    _same_tables(got, want)


@pytest.mark.parametrize("rows", [20, 5000])
def test_tables_bad_requests_keep_what_they_have(rows):
    rng = np.random.default_rng(rows)
    c = _tables_case(rng, 40, 5, 32, 100, rows, refuse=True)
    _log(f"[tables] bad requests, rows={rows}")
    got = _run_tables(c, 40, 32, rows, False)
    want = kvq8.build_block_tables(c["want"], 32, c["bt"], c["held"], c["stack"], c["free"], c["ro"],
                                   c["start"], rows)
    assert got["status"] & st.BAD_OFFSETS
    _same_tables(got, want)


@pytest.mark.parametrize("free", [-1, 1 << 20])
def test_tables_bad_stack_changes_nothing(free):
    rng = np.random.default_rng(1)
    c = _tables_case(rng, 10, 4, 32, 6, 30)
    c["free"] = free
    _log(f"[tables] stack of {free}")
    got = _run_tables(c, 10, 32, 30, False)
    want = kvq8.build_block_tables(c["want"], 32, c["bt"], c["held"], c["stack"], free, c["ro"],
                                   c["start"], 30)
    assert got["status"] & st.BAD_OFFSETS
    assert np.array_equal(got["block_table"], c["bt"]) and np.array_equal(got["num_held"], c["held"])
    _same_tables(got, want)


def test_tables_without_slot_map_and_with_bad_offsets():
    rng = np.random.default_rng(4)
    c = _tables_case(rng, 12, 4, 32, 20, 40)
    got = _run_tables(c, 12, 32, 0, False, slot_map=False)
    want = kvq8.build_block_tables(c["want"], 32, c["bt"], c["held"], c["stack"], c["free"])
    _same_tables(got, want)
    # offsets that decrease or leave the rows: every entry is written, none out of bounds
    for ro in (np.full(13, 7), np.arange(13)[::-1] * 3, np.full(13, -4), np.full(13, 1 << 30)):
        for rows in (40, 5000):
            c["ro"] = ro.astype(np.int32)
            got = _run_tables(c, 12, 32, rows, False)
            assert np.all(got["slot_map"] >= -1)


# ---- attention --------------------------------------------------------------

def _tree(rng, n, W):
    """Random ancestor masks of n slots."""
    m = np.zeros((n, W), np.uint32)
    for j in range(n):
        if j:
            m[j] = m[rng.integers(max(0, j - 5), j)]
        m[j, j >> 5] |= np.uint32(1 << (j & 31))
    return m


def _attn_case(rng, hq, hkv, slots, plens, ps, fmt, q_scale=1.0, scales=None, extra_pages=2, spare=3):
    R = len(plens)
    cap = sum(slots) + spare
    W = (max(slots) + 31) // 32 if max(slots) else 1
    mask = np.zeros((cap, W), np.uint32)
    qo = np.zeros(R + 1, np.int32)
    qo[1:] = np.cumsum(slots)
    for r in range(R):
        mask[qo[r]:qo[r + 1]] = _tree(rng, slots[r], W)
    _, pages, bt = _slots_of(plens, [0] * R, ps, rng, extra_pages)
    cache = _empty_cache(rng, pages, hkv, ps)
    for i in range(2):  # tokens that requests hold are finite, the others are any bytes
        cache[2 + i] = (np.exp2(rng.integers(-9, -5, cache[2 + i].shape)) if scales is None
                        else rng.uniform(*scales, cache[2 + i].shape)).astype(np.float32)
        for r in range(R):
            for p in range(plens[r]):
                cache[i][bt[r, p // ps], :, p % ps] = kvq8.encode8(
                    rng.standard_normal((hkv, 128)) * (100.0 if fmt == kvq8.E4M3 else 9000.0), fmt)
    if fmt == kvq8.E5M2:
        for i in range(2):
            cache[2 + i] *= np.float32(2.0 ** -7)
    return dict(R=R, hq=hq, hkv=hkv, cap=cap, W=W, ps=ps, fmt=fmt, q=_bf(rng.standard_normal((cap, hq, 128)) * q_scale),
                kn=_bf(rng.standard_normal((cap, hkv, 128))), vn=_bf(rng.standard_normal((cap, hkv, 128))),
                cache=cache, bt=bt, plen=np.array(plens, np.int32), qo=qo, mask=mask, scale=128 ** -0.5)


def _attn_args(c, out, lse, ws, status):
    return (_dev(c["q"]), _dev(c["kn"]), _dev(c["vn"]), c["fmt"], *[_dev(a) for a in c["cache"]], c["ps"],
            _dev(c["bt"]), _dev(c["plen"]), _dev(c["qo"]), _dev(c["mask"]), c["W"], c["R"], c["cap"], c["hq"],
            c["hkv"], 128, c["scale"], out, lse, ws, status)


def _attn_buffers(c):
    import torch
    import paper_2604_09603_amd as pkg
    from paper_2604_09603_amd.step import _aligned_workspace
    out = torch.full((c["cap"], c["hq"], 128), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    lse = torch.full((c["cap"], c["hq"]), float("nan"), dtype=torch.float32, device="cuda:0")
    ws = _aligned_workspace(pkg.tree_verify_attn_paged_q8_workspace_size(
        c["R"], c["cap"], c["hq"], c["hkv"], c["bt"].shape[1]), "cuda:0")
    ws.fill_(0xCD)
    return out, lse, ws, _zeros(1)


def _run_attn(c):
    import torch
    import paper_2604_09603_amd as pkg
    out, lse, ws, status = _attn_buffers(c)
    pkg.echo_tree_verify_attn_paged_q8(*_attn_args(c, out, lse, ws, status))
    torch.cuda.synchronize()
    return out.float().cpu().numpy(), lse.cpu().numpy(), int(status.item())


def _check_attn(c, out, lse, status, want_status=0):
    """Error bounds, per element.  With w a row's weights, v its values, o its output:
    * the rounding of each w to bf16 (at most 2^-8 of it), sums of the rounded ones: the output
      moves by at most 2^-8 / (1 - 2^-8) of the mean |v - o|;
    * a score's fp32 error: 129 additions and products of 2^-24 each on sum |q k|, twice that for the
      scales' products and the exponent's fma; an exponential's 2^-22: a relative error of w, on the
      same mean;
    * partial sums in fp16: half a step is at most 2^-11 of the row's largest part, and parts are
      convex combinations too, at most vmax;
    * fp32 sums over up to 4000 keys: 2^-24 * 64 of vmax (a chain is shorter than 64 tiles of 64 keys);
    * the output's own rounding, 2^-8 of it."""
    ref = kvq8.tree_verify_attn_paged_q8(c["q"], c["kn"], c["vn"], c["fmt"], *c["cache"], c["bt"], c["plen"],
                                         c["qo"], c["mask"], c["hq"], c["hkv"], c["scale"])
    assert status == ref["status"] == want_status
    nq = int(c["qo"][-1])
    live = ~np.isnan(ref["lse"])
    assert np.all(np.isnan(out[:nq]) == ~live[..., None]), "rows written or not"
    assert np.all(np.isnan(out[nq:])) and np.all(np.isnan(lse[nq:]))
    o, l = out[:nq][live].astype(np.float64), lse[:nq][live].astype(np.float64)
    ro, rl = ref["out"][live], ref["lse"][live]
    dz = ref["zabs"][live][:, None] * (2 * 129 * 2.0 ** -24)
    tol = (ref["dev"][live] * (2.0 ** -8 / (1 - 2.0 ** -8) + dz + 2.0 ** -22)
           + ref["vmax"][live][:, None] * (2.0 ** -11 + 2.0 ** -18))
    tol = tol * (1 + 2.0 ** -7) + np.abs(ro) * 2.0 ** -8
    err = np.abs(o - ro)
    assert np.all(err <= tol), f"off by {np.nanmax(err / np.maximum(tol, 1e-300)):.3f} of the bound"
    empty = np.isneginf(rl)
    assert np.array_equal(np.isneginf(l), empty) and np.all(o[empty] == 0)
    f = ~empty
    assert np.all(np.abs(l[f] - rl[f]) <= dz[f, 0] + 2.0 ** -18 + np.abs(rl[f]) * 2.0 ** -22)


CASES = [
    # hq, hkv, slots, prefixes, page
    (1, 1, [1], [0], 32), (1, 1, [1], [1], 32), (8, 8, [1, 1, 1], [31, 32, 33], 32),
    (8, 1, [3, 1], [64, 65], 64), (16, 2, [1, 5, 2], [0, 700, 95], 64),
    (32, 8, [5, 1, 4, 7], [130, 1, 255, 40], 128), (64, 4, [1, 3, 0, 4], [96, 300, 50, 0], 32),
    (64, 4, [5, 9], [500, 33], 256), (40, 5, [2, 13], [129, 260], 64),
    (4, 4, [33, 64, 65], [10, 0, 70], 32), (8, 2, [100, 17], [31, 100], 64), (12, 3, [6] * 9, [37 * i for i in range(9)], 32)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_matches_oracle(case, fmt):
    hq, hkv, slots, plens, ps = CASES[case]
    rng = np.random.default_rng(100 * case + fmt)
    c = _attn_case(rng, hq, hkv, slots, plens, ps, fmt)
    _log(f"[attn q8] {CASES[case]} fmt={fmt}")
    _check_attn(c, *_run_attn(c))


def test_attention_long_prefixes():
    """Units that many waves share, and several requests in one wave's range."""
    rng = np.random.default_rng(9)
    c = _attn_case(rng, 8, 2, [3, 1, 1], [3999, 2048, 1], 64, kvq8.E4M3)
    _log("[attn q8] long prefixes")
    _check_attn(c, *_run_attn(c))


def test_attention_many_requests():
    rng = np.random.default_rng(10)
    R = 1500
    c = _attn_case(rng, 4, 2, [1] * R, rng.integers(0, 40, R).tolist(), 32, kvq8.E4M3)
    _log("[attn q8] 1500 requests")
    _check_attn(c, *_run_attn(c))


def test_attention_largest_batch():
    """As many requests as a call takes, some with heads of more than 128 rows."""
    rng = np.random.default_rng(19)
    R = 4095
    slots = [9 if r % 500 == 7 else 1 for r in range(R)]
    c = _attn_case(rng, 16, 1, slots, rng.integers(0, 20, R).tolist(), 32, kvq8.E4M3)
    _log("[attn q8] 4095 requests")
    _check_attn(c, *_run_attn(c))


@pytest.mark.parametrize("q_scale", [0.0, 30.0])
def test_attention_flat_and_peaked_rows(q_scale):
    rng = np.random.default_rng(12)
    c = _attn_case(rng, 16, 2, [4, 2], [400, 77], 64, kvq8.E4M3, q_scale=q_scale)
    _log(f"[attn q8] q_scale={q_scale}")
    _check_attn(c, *_run_attn(c))


def test_attention_any_scales():
    rng = np.random.default_rng(13)
    c = _attn_case(rng, 8, 4, [2, 3], [200, 70], 32, kvq8.E4M3, scales=(0.001, 0.02))
    c["cache"][3] *= np.exp2(rng.integers(-20, 3, c["cache"][3].shape)).astype(np.float32)
    _log("[attn q8] scales of any value")
    _check_attn(c, *_run_attn(c))


def test_attention_empty_masks():
    """Rows that see nothing: no prefix and no bit; and rows that see the prefix alone."""
    rng = np.random.default_rng(14)
    c = _attn_case(rng, 8, 2, [3, 2, 40], [0, 50, 0], 32, kvq8.E4M3)
    c["mask"][[0, 2, 3, 4, 5, 20, 44]] = 0
    _log("[attn q8] empty masks")
    _check_attn(c, *_run_attn(c))


@pytest.mark.parametrize("big", [False, True])
def test_attention_skips_bad_requests(big):
    """A missing page, a page past the pool, a length past the table, decreasing offsets; with
    small tables (checked by the plan) and large ones.  Ids past a prefix don't count."""
    rng = np.random.default_rng(15)
    c = _attn_case(rng, 8, 2, [2, 3, 1, 2, 1, 2], [70, 40, 33, 90, 20, 0], 32, kvq8.E4M3)
    if big:
        c["bt"] = np.pad(c["bt"], ((0, 0), (0, 3000)), constant_values=-1)
    pages = c["cache"][0].shape[0]
    c["bt"][1, 1] = -1
    c["bt"][3, 2] = pages
    c["bt"][4, 1:] = pages + 5
    c["plen"][2] = c["bt"].shape[1] * 32 + 1
    _log(f"[attn q8] bad requests big={big}")
    out, lse, status = _run_attn(c)
    assert status == st.BAD_OFFSETS
    c["plen"][2] = -1  # (the oracle's form of a length that cannot be)
    _check_attn(c, out, lse, status, st.BAD_OFFSETS)
    c["plen"][:] = -3  # nothing left to do: nothing is written
    out, lse, status = _run_attn(c)
    assert status == st.BAD_OFFSETS and np.isnan(out).all() and np.isnan(lse).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_attention_scores_that_cancel(fmt):
    """Two products of a score are large and cancel: what is left is still held in 32 bits."""
    rng = np.random.default_rng(16)
    c = _attn_case(rng, 8, 2, [1, 2, 1, 3], [1, 33, 2, 64], 32, fmt)
    q = c["q"].astype(np.uint32).__lshift__(16).view(np.float32).copy()
    q[..., 0] = q[..., 1] = 128.0
    c["q"] = _bf(q)
    top = 0x7E if fmt == kvq8.E4M3 else 0x78  # 448; 32768
    c["cache"][0][..., 0], c["cache"][0][..., 1] = top, top | 0x80
    c["mask"][[0, 3]] = 0
    _log(f"[attn q8] scores that cancel fmt={fmt}")
    _check_attn(c, *_run_attn(c))


def test_attention_heads_of_every_size_in_one_batch():
    """Requests with up to 32, 64, 128 and more rows per head side by side, some without work."""
    rng = np.random.default_rng(17)
    c = _attn_case(rng, 32, 2, [1, 2, 3, 0, 4, 5, 8, 9, 17, 1, 33], [700, 64, 333, 90, 1, 400, 31, 0, 129, 0, 95],
                   64, kvq8.E4M3)
    _log("[attn q8] heads of every size")
    _check_attn(c, *_run_attn(c))


@pytest.mark.parametrize("R,width", [(1024, 32), (1025, 32), (1024, 33), (4, 8300)])
def test_attention_page_checks_of_every_size(R, width):
    """Block tables just small enough for one workgroup's check, and just too large; bad ids in
    the first, a middle and the last request."""
    rng = np.random.default_rng(18)
    plens = rng.integers(1, 34, R).tolist()
    plens[0] = plens[R // 2] = plens[R - 1] = 64
    c = _attn_case(rng, 2, 1, [1] * R, plens, 32, kvq8.E4M3)
    pad = width - c["bt"].shape[1]
    c["bt"] = np.pad(c["bt"], ((0, 0), (0, pad)), constant_values=-1)
    c["bt"][0, 1] = -1
    c["bt"][R // 2, 0] = c["cache"][0].shape[0]
    c["bt"][R - 1, 1] = -2 ** 31
    _log(f"[attn q8] page checks R={R} width={width}")
    out, lse, status = _run_attn(c)
    _check_attn(c, out, lse, status, st.BAD_OFFSETS)
    assert np.isnan(lse[[0, R // 2, R - 1]]).all() and np.isfinite(lse[1]).all()


@pytest.mark.parametrize("width", [4, 600])
def test_attention_pages_of_requests_without_slots_count(width):
    """A request that has nothing to verify writes nothing, but its missing page is reported."""
    rng = np.random.default_rng(20)
    c = _attn_case(rng, 8, 2, [2, 0, 1], [40, 70, 33], 32, kvq8.E4M3)
    c["bt"] = np.pad(c["bt"], ((0, 0), (0, width - c["bt"].shape[1])), constant_values=-1)
    _log(f"[attn q8] no slots, width={width}")
    _check_attn(c, *_run_attn(c))
    c["bt"][1, 2] = -1
    _check_attn(c, *_run_attn(c), st.BAD_OFFSETS)


def test_attention_widest_block_table():
    """One request whose row of the block table has 20 million entries."""
    rng = np.random.default_rng(21)
    c = _attn_case(rng, 4, 2, [2], [77], 32, kvq8.E4M3)
    c["bt"] = np.pad(c["bt"], ((0, 0), (0, 20_000_000)), constant_values=-1)
    _log("[attn q8] 20 million entries")
    _check_attn(c, *_run_attn(c))


def test_attention_without_lse_and_on_a_stream():
    import torch
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(16)
    c = _attn_case(rng, 16, 4, [3, 1], [260, 99], 64, kvq8.E5M2)
    ref, _, _ = _run_attn(c)
    # two calls at once, each with buffers of its own
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    runs = []
    for s in side:
        bufs = _attn_buffers(c)
        runs.append((bufs, _attn_args(c, bufs[0], None, *bufs[2:])))
    torch.cuda.synchronize()
    _log("[attn q8] two streams")
    for s, (_, args) in zip(side, runs):
        pkg.echo_tree_verify_attn_paged_q8(*args, stream=s)
    torch.cuda.synchronize()
    for bufs, _ in runs:
        got = bufs[0].float().cpu().numpy()
        assert np.array_equal(got, ref, equal_nan=True)


def test_two_captured_calls_share_a_workspace():
    """Graphs of two batches with one workspace, replayed in turn: each replay is its eager call."""
    import torch
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(22)
    batches = [_attn_case(rng, 32, 2, [1, 9, 3], [500, 40, 999], 64, kvq8.E4M3),
               _attn_case(rng, 8, 8, [1] * 5, [10, 300, 0, 77, 1], 32, kvq8.E5M2)]
    bufs = [_attn_buffers(c) for c in batches]
    ws = max((b[2] for b in bufs), key=lambda w: w.numel())
    args = [_attn_args(c, b[0], b[1], ws, b[3]) for c, b in zip(batches, bufs)]
    _log("[attn q8] two graphs")

    def fetch(b):
        torch.cuda.synchronize()
        return b[0].view(torch.int16).cpu().numpy(), b[1].view(torch.int32).cpu().numpy()

    eager, graphs = [], []
    for a, b in zip(args, bufs):
        pkg.echo_tree_verify_attn_paged_q8(*a)
        eager.append(fetch(b))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            pkg.echo_tree_verify_attn_paged_q8(*a)
    for i in (0, 1, 1, 0, 1, 0):
        for b in bufs:
            b[0].fill_(float("nan"))
            b[1].fill_(float("nan"))
        graphs[i].replay()
        for x, y in zip(fetch(bufs[i]), eager[i]):
            assert np.array_equal(x, y), i


def test_offsets_past_32_bits():
    """A pool of 4.6 GB per tensor: its last pages are written and read."""
    import torch
    rng = np.random.default_rng(17)
    hkv, ps = 8, 256
    c = _attn_case(rng, 8, hkv, [1, 2], [300, 31], ps, kvq8.E4M3)
    pages = 17600
    assert pages * hkv * ps * 128 > 1 << 32
    n = c["cache"][0].shape[0]
    big = [torch.zeros((pages, *a.shape[1:]), dtype=_dev(a).dtype, device="cuda:0") for a in c["cache"]]
    T = 100
    x = _values(rng, T, hkv, 128)
    slots = np.arange(40, 40 + T, dtype=np.int64) + (pages - 1) * ps
    for t, a in zip(big, c["cache"]):
        t[pages - n:] = _dev(a)
    import paper_2604_09603_amd as pkg
    out, lse, ws, status = _attn_buffers(c)
    args = list(_attn_args(c, out, lse, ws, status))
    args[4:8] = big
    args[9] = _dev(np.where(c["bt"] >= 0, c["bt"] + pages - n, -1).astype(np.int32))
    _log("[q8] a pool past 4 GB")
    pkg.echo_tree_verify_attn_paged_q8(*args)
    _check_attn(c, out.float().cpu().numpy(), lse.cpu().numpy(), int(status.item()))
    _store(_dev(x), _dev(x), _dev(slots), kvq8.E4M3, big, ps)
    small = [a[-1:].copy() for a in c["cache"]]
    *want, _ = kvq8.store_kv(x, x, slots - (pages - 1) * ps, kvq8.E4M3, *small)
    for i in range(2):
        _same_bytes(big[i][-1:].cpu().numpy(), want[i], kvq8.E4M3, f"tensor {i}")
        assert not big[i][:100].any()


# ---- together ---------------------------------------------------------------

def _serving_run(fmt, steps, ps=32):
    """Prompts into a fresh cache, then steps of pages, attention, acceptance and commit, on the
    GPU; every output is returned, and the host's copy of what each call saw."""
    import torch
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(21 + fmt)
    R, hq, hkv, most, depth = 5, 8, 2, 12, 4
    total = 40
    prompts = np.array([70, 1, 33, 64, 12], np.int32)
    cache = _empty_cache(rng, total, hkv, ps)
    dev = [_dev(a) for a in cache]
    bt, stack = _dev(np.full((R, most), -1, np.int32)), _dev(rng.permutation(total).astype(np.int32))
    held, free, status = _zeros(R), _dev(np.array([total], np.int32)), _zeros(1)
    plen = _zeros(R)
    ro = np.zeros(R + 1, np.int32)
    ro[1:] = np.cumsum(prompts)
    T = int(ro[-1])
    k, v = _values(rng, T, hkv, 128), _values(rng, T, hkv, 128)
    sm = torch.zeros(T + 5, dtype=torch.int64, device="cuda:0")
    pkg.echo_build_block_tables(_dev(prompts), R, ps, bt, held, held, stack, free, free,
                                row_offsets=_dev(ro), row_start=plen, slot_map=sm, status=status)
    pad = np.zeros((5, hkv, 128), np.uint16)
    _store(_dev(np.concatenate([k, pad])), _dev(np.concatenate([v, pad])), sm, fmt, dev, ps, status)
    plen.copy_(_dev(prompts))
    log = [dict(kind="store", k=k, v=v, slots=sm.cpu().numpy()[:T], cache=[t.cpu().numpy() for t in dev])]
    slots = [3, 1, 5, 2, 4]
    cap = sum(slots)
    qo = np.zeros(R + 1, np.int32)
    qo[1:] = np.cumsum(slots)
    W = 1
    mask = np.concatenate([_tree(rng, n, W) for n in slots])
    for step in range(steps):
        c = dict(R=R, hq=hq, hkv=hkv, cap=cap, W=W, ps=ps, fmt=fmt, qo=qo, mask=mask, scale=128 ** -0.5,
                 q=_bf(rng.standard_normal((cap, hq, 128))), kn=_values(rng, cap, hkv, 128),
                 vn=_values(rng, cap, hkv, 128))
        want = plen + depth + 1
        pkg.echo_build_block_tables(want, R, ps, bt, held, held, stack, free, free, status=status)
        c.update(bt=bt.cpu().numpy(), plen=plen.cpu().numpy(), cache=[t.cpu().numpy() for t in dev])
        out, lse, ws, _ = _attn_buffers(c)
        kn, vn = _dev(c["kn"]), _dev(c["vn"])
        pkg.echo_tree_verify_attn_paged_q8(_dev(c["q"]), kn, vn, fmt, *dev, ps, bt, plen, _dev(qo),
                                           _dev(mask), W, R, cap, hq, hkv, 128, c["scale"], out, lse, ws,
                                           status=status)
        acc_len = np.minimum(rng.integers(0, depth + 1, R), np.array(slots) - 1).astype(np.int32)
        acc = np.full((R, depth), -1, np.int32)
        for r in range(R):
            acc[r, :acc_len[r]] = qo[r] + 1 + np.arange(acc_len[r])
        pkg.echo_commit_kv_q8(_dev(qo), _dev(acc_len), _dev(acc), depth, kn, vn, R, cap, hkv, 128, fmt,
                              *dev, ps, bt, plen, plen, status=status)
        c.update(kind="step", out=out.float().cpu().numpy(), lse=lse.cpu().numpy(), acc_len=acc_len, acc=acc,
                 after=[t.cpu().numpy() for t in dev], new_len=plen.cpu().numpy())
        log.append(c)
    assert int(status.item()) == 0
    return log, cache


@pytest.mark.parametrize("fmt", FMTS)
def test_prompts_then_steps(fmt):
    log, cache = _serving_run(fmt, 6)
    *want, _ = kvq8.store_kv(log[0]["k"], log[0]["v"], log[0]["slots"], fmt, *cache)
    assert len(set(log[0]["slots"].tolist())) == len(log[0]["slots"])
    for i in range(4):
        _same_bytes(log[0]["cache"][i], want[i], fmt, i) if i < 2 else np.testing.assert_array_equal(
            log[0]["cache"][i], want[i])
    for n, c in enumerate(log[1:]):
        _log(f"[q8 step] fmt={fmt} step {n}")
        _check_attn(c, c["out"], c["lse"], 0)
        *want, new_len, status = kvq8.commit_kv_q8(c["qo"], c["acc_len"], c["acc"], c["kn"], c["vn"], fmt,
                                                   *c["cache"], c["bt"], c["plen"])
        assert status == 0 and np.array_equal(new_len, c["new_len"])
        for i in range(4):
            _same_bytes(c["after"][i], want[i], fmt, i) if i < 2 else np.testing.assert_array_equal(
                c["after"][i], want[i])


def test_captured_step_replays():
    """Pages, store, attention and commit captured in one graph and replayed on changing
    inputs, with eager work between the replays: every replay equals the eager calls."""
    import torch
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(33)
    fmt, ps = kvq8.E4M3, 64
    c = _attn_case(rng, 16, 4, [3, 2, 4], [100, 63, 250], ps, fmt, extra_pages=9, spare=0)
    R, cap, hkv, depth = c["R"], c["cap"], c["hkv"], 4
    held = np.array([-(-int(p) // ps) for p in c["plen"]], np.int32)
    bt0 = np.pad(c["bt"], ((0, 0), (0, 2)), constant_values=-1)
    c["bt"] = bt0
    pages = c["cache"][0].shape[0]
    used = {int(x) for x in bt0[bt0 >= 0]}
    stack0 = np.array([p for p in range(pages) if p not in used] + [-1] * len(used), np.int32)
    ro = np.array([0, 1, 2, 3], np.int32)
    names = ("q", "kn", "vn")

    def fresh(seed):
        g = np.random.default_rng(seed)
        return dict(q=_bf(g.standard_normal(c["q"].shape)), kn=_values(g, cap, hkv, 128),
                    vn=_values(g, cap, hkv, 128), acc=g.integers(0, 2, R).astype(np.int32))

    d = dict(cache=[_dev(a) for a in c["cache"]], bt=_dev(bt0), stack=_dev(stack0), held=_dev(held),
             free=_dev(np.array([pages - len(used)], np.int32)), plen=_dev(c["plen"]), qo=_dev(c["qo"]),
             mask=_dev(c["mask"]), ro=_dev(ro), new=_zeros(R), held_out=_zeros(R), free_out=_zeros(1),
             want=_dev(c["plen"] + depth + 2), acc_len=_zeros(R), acc=_dev(np.stack(
                 [c["qo"][:-1] + 1] + [np.full(R, -1)] * (depth - 1), 1).astype(np.int32)))
    for n in names:
        d[n] = _dev(c[n])
    d["sm"] = torch.zeros(R + 2, dtype=torch.int64, device="cuda:0")
    out, lse, ws, status = _attn_buffers(c)
    init = {n: ([t.clone() for t in d[n]] if n == "cache" else d[n].clone()) for n in d}

    def step():
        pkg.echo_build_block_tables(d["want"], R, ps, d["bt"], d["held"], d["held_out"], d["stack"], d["free"],
                                    d["free_out"], row_offsets=d["ro"], row_start=d["plen"], slot_map=d["sm"],
                                    status=status)
        pkg.echo_tree_verify_attn_paged_q8(d["q"], d["kn"], d["vn"], fmt, *d["cache"], ps, d["bt"], d["plen"],
                                           d["qo"], d["mask"], c["W"], R, cap, c["hq"], hkv, 128, c["scale"],
                                           out, lse, ws, status=status)
        pkg.echo_store_kv_q8(d["kn"], d["vn"], d["sm"], R + 2, hkv, 128, fmt, *d["cache"], ps, status=status)
        pkg.echo_commit_kv_q8(d["qo"], d["acc_len"], d["acc"], depth, d["kn"], d["vn"], R, cap, hkv, 128, fmt,
                              *d["cache"], ps, d["bt"], d["plen"], d["new"], status=status)

    def reset(x):
        for n in init:
            if n == "cache":
                for t, u in zip(d[n], init[n]):
                    t.copy_(u)
            else:
                d[n].copy_(init[n])
        for n in names:
            d[n].copy_(_dev(x[n]))
        d["acc_len"].copy_(_dev(x["acc"]))
        out.fill_(float("nan"))
        lse.fill_(float("nan"))

    def fetch():
        torch.cuda.synchronize()
        return [t.cpu().numpy() for t in (out.view(torch.int16), lse.view(torch.int32), d["bt"], d["held_out"],
                                          d["free_out"], d["sm"], d["new"], *d["cache"], status)]

    eager = []
    for seed in range(3):
        reset(fresh(seed))
        step()
        eager.append(fetch())
    reset(fresh(0))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (1, 0, 2, 1, 2):
        reset(fresh(i))
        x = torch.randn(128, 128, device="cuda:0")
        (x @ x).sum().item()
        graph.replay()
        for k, (a, b) in enumerate(zip(fetch(), eager[i])):
            assert np.array_equal(a, b), (i, k)
    assert int(status.item()) == 0
