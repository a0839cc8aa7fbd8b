"""GPU parity of rotary positions and of the latent cache's writers against the oracle, within
bounds per element that follow from the documented roundings."""
import numpy as np
import pytest

from oracle import latent, status as st
from synth.batch import f32_to_bf16_bits
from tests import gpu_common as gc

pytestmark = pytest.mark.gpu
LAYOUTS = (latent.HALF, latent.INTERLEAVED)


@pytest.fixture(autouse=True)
def _need_gpu():
    gc.require_gpu()


def _log(msg):
    print(msg, flush=True)


def _dev(a, dtype=None):
    import torch
    a = np.ascontiguousarray(a if dtype is None else np.asarray(a, dtype))
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).to("cuda:0").view(torch.bfloat16)
    if a.dtype == np.uint32:
        a = a.view(np.int32)
    return torch.from_numpy(a).to("cuda:0")


def _bits(t):
    """The bits of a bf16 tensor."""
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _bf(x):
    return f32_to_bf16_bits(np.ascontiguousarray(x, np.float32)).reshape(np.shape(x))


f64 = latent.bf16_to_f64


def _zeros(*s):
    import torch
    return torch.zeros(s, dtype=torch.int32, device="cuda:0")


# ---- rotary positions ---------------------------------------------------------

def _rotated_ok(got, x, positions, f, scale, layout):
    """Bounds per element: the output's rounding, 2^-8 of it; an angle's error of 2^-26 of a turn
    (its fraction in fp32) and of 2^-51 of the position (products in 64 bits, here and in
    the oracle), in radians, and 2^-22 for the cosine and sine, 3 * 2^-24 for their
    scale, the products and the sum, on |a| + |b|."""
    want = latent.rotate(x, positions, f, scale, layout)
    mag = latent.rotate(np.abs(x), np.zeros(len(x)), f, 1.0, layout)
    h = x.shape[-1] // 2
    a, b = (mag[..., 0::2], mag[..., 1::2]) if layout else (mag[..., :h], mag[..., h:])
    both = np.stack([a + b, a + b], -1).reshape(x.shape) if layout else np.concatenate([a + b, a + b], -1)
    far = np.abs(np.asarray(positions, np.float64)).reshape((-1,) + (1,) * (x.ndim - 1))
    turn = 2 * np.pi * 2.0 ** -26 + far * 2.0 ** -51 + 2.0 ** -22 + 3 * 2.0 ** -24
    tol = np.abs(want) * 2.0 ** -8 + abs(scale) * both * turn * (1 + 2.0 ** -8)
    err = np.abs(f64(got) - want)
    assert np.all(err <= tol), f"off by {(err / np.maximum(tol, 1e-300)).max():.3f} of the bound"


def _rope(q, q_out, k, k_out, pos, f, scale, layout, **kw):
    import paper_2604_09603_amd as pkg
    hk = 0 if k is None else k.shape[1]
    pkg.echo_rope(q, q_out, k, k_out, pos, q.shape[0], q.shape[1], hk, q.shape[2], layout, f, scale, **kw)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rows,hq,hk,rot,scaling", [
    (1, 1, 1, 2, "plain"), (3, 5, 2, 6, "linear"), (7, 64, 4, 128, "plain"), (33, 12, 3, 24, "smooth"),
    (130, 32, 8, 128, "smooth"), (5, 128, 1, 64, "bands"), (2, 3, 0, 1024, "base"), (9, 7, 1, 80, "bands"),
    (513, 2, 1, 64, "plain"), (4, 1, 300, 16, "plain"), (3, 2, 2, 1022, "plain")])
def test_rope_matches_oracle(rows, hq, hk, rot, scaling, layout):
    import torch
    rng = np.random.default_rng(rows * 1000 + rot)
    f, scale = latent.frequencies(rot, 10000.0, scaling, 8.0, 4096.0, 1.0, 32.0)
    pos = rng.integers(-(1 << 20), 1 << 20, rows)
    pos[0] = 0
    q, k = _bf(rng.standard_normal((rows, hq, rot))), _bf(rng.standard_normal((rows, hk, rot)))
    _log(f"[rope] rows={rows} heads={hq}/{hk} rot={rot} {scaling} layout={layout}")
    qd, kd = _dev(q), _dev(k) if hk else None
    qo, ko = torch.zeros_like(qd), torch.zeros_like(kd) if hk else None
    p, fd = _dev(pos, np.int32), _dev(f)
    _rope(qd, qo, kd, ko, p, fd, scale, layout)
    _rotated_ok(_bits(qo), f64(q), pos, f, float(np.float32(scale)), layout)
    assert np.array_equal(_bits(qd), q)
    if hk:
        _rotated_ok(_bits(ko), f64(k), pos, f, float(np.float32(scale)), layout)
    _rope(qd, qd, kd, kd, p, fd, scale, layout)  # in place
    assert torch.equal(qd, qo) and (not hk or torch.equal(kd, ko))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("shift", [0, 1])
def test_rope_part_of_wider_heads(layout, shift):
    """The rotated part inside wider heads, into the end of another layout, heads outermost: the
    other dims stay as they are.  shift: rows that are not 16-byte aligned."""
    import torch
    rng = np.random.default_rng(3)
    T, h, rot = 37, 6, 32
    x = _bf(rng.standard_normal((T, h, 100 + rot)))
    pos, (f, _) = rng.integers(0, 9000, T), latent.frequencies(rot, 10000.0)
    xd = _dev(x)
    y = torch.full((h, T, 72 + rot), 7.0, dtype=torch.bfloat16, device="cuda:0")
    _log(f"[rope] part of a head, layout={layout} shift={shift}")
    # (element 96 of 132 is 8-byte aligned in odd heads: pair by pair; the output is aligned)
    out = y.transpose(0, 1)[..., 64 + shift:64 + shift + rot]
    _rope(xd[..., 96:96 + rot], out, None, None, _dev(pos, np.int32), _dev(f), 1.0, layout)
    _rotated_ok(_bits(out), f64(x[..., 96:96 + rot]), pos, f, 1.0, layout)
    rest = torch.cat([y[..., :64 + shift], y[..., 64 + shift + rot:]], -1)
    assert torch.all(rest == 7.0) and np.array_equal(_bits(xd), x)


def test_rope_same_bits_aligned_or_not():
    import torch
    rng = np.random.default_rng(4)
    x = _dev(_bf(rng.standard_normal((50, 9, 64))))
    odd = torch.zeros((50, 9, 67), dtype=torch.bfloat16, device="cuda:0")[..., 1:65]
    odd.copy_(x)
    p, f = _dev(rng.integers(0, 1 << 17, 50), np.int32), _dev(latent.frequencies(64, 1e4)[0])
    for layout in LAYOUTS:
        a, b = torch.zeros_like(x), torch.zeros((50, 9, 67), dtype=torch.bfloat16, device="cuda:0")[..., 1:65]
        _rope(x, a, None, None, p, f, 1.25, layout)
        _rope(odd, b, None, None, p, f, 1.25, layout)
        assert torch.equal(a, b)


def test_rope_far_positions_and_repeated_heads():
    """The ends of the positions' range; one row of keys read by every head (stride 0)."""
    import torch
    rng = np.random.default_rng(5)
    pos = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, 2 ** 24 + 1, 1, 0], np.int64)
    x, (f, _) = _bf(rng.standard_normal((6, 1, 64))), latent.frequencies(64, 10000.0)
    many = _dev(x).expand(6, 5, 64)
    out = torch.zeros((6, 5, 64), dtype=torch.bfloat16, device="cuda:0")
    for layout in LAYOUTS:
        _rope(many, out, None, None, _dev(pos, np.int32), _dev(f), 1.0, layout)
        for h in range(5):
            _rotated_ok(_bits(out[:, h:h + 1]), f64(x), pos, f, 1.0, layout)


def test_rope_rows_that_exist():
    import torch
    rng = np.random.default_rng(6)
    x = _dev(_bf(rng.standard_normal((20, 3, 32))))
    p, f = _dev(np.arange(20), np.int32), _dev(latent.frequencies(32, 1e4)[0])
    whole = torch.zeros_like(x)
    _rope(x, whole, None, None, p, f, 1.0, 0)
    for n, bits in [(0, 0), (1, 0), (13, 0), (20, 0), (21, st.BAD_OFFSETS), (-1, st.BAD_OFFSETS)]:
        out, status = torch.full_like(x, 5.0), _zeros(1)
        _rope(x, out, None, None, p, f, 1.0, 0, row_count=_dev([n], np.int32), status=status)
        live = n if bits == 0 else 0
        assert int(status.item()) == bits
        assert torch.equal(out[:live], whole[:live]) and torch.all(out[live:] == 5.0)


def test_rope_gradient():
    """The gradient of sum(g rope(x)) is rope(g) with negated frequencies: against differences
    of the oracle along random directions, and against the formula."""
    import torch
    rng = np.random.default_rng(7)
    g, pos = _bf(rng.standard_normal((11, 4, 64))), rng.integers(0, 1 << 16, 11)
    f, scale = latent.frequencies(64, 10000.0, "bands", 40.0, 4096.0)
    for layout in LAYOUTS:
        out = torch.zeros((11, 4, 64), dtype=torch.bfloat16, device="cuda:0")
        _rope(_dev(g), out, None, None, _dev(pos, np.int32), _dev(-f), scale, layout)
        s = float(np.float32(scale))
        _rotated_ok(_bits(out), f64(g), pos, -f, s, layout)
        # the loss is linear: the difference along e is exact up to the gradient's own rounding
        e = rng.standard_normal(g.shape)
        diff = (f64(g) * (latent.rotate(e, pos, f, s, layout) - latent.rotate(-e, pos, f, s, layout))).sum() / 2
        grad = f64(_bits(out))
        assert abs((grad * e).sum() - diff) <= (np.abs(grad * e)).sum() * 2.0 ** -7


# ---- the writers ------------------------------------------------------------------

def _slots_of(lens, starts, ps, rng, spare=2):
    """Slots of rows [start, start + len) of each request over shuffled pages; the pool's pages."""
    npg = [-(-(s + n) // ps) for s, n in zip(starts, lens)]
    perm = rng.permutation(sum(npg) + spare)
    at, slots = 0, []
    for r, (n, s) in enumerate(zip(lens, starts)):
        p = np.arange(s, s + n)
        slots.append(perm[at + p // ps].astype(np.int64) * ps + p % ps)
        at += npg[r]
    return np.concatenate(slots), len(perm)


def _store(kv, weight, pos, f, scale, layout, new=None, slots=None, pages=None, ps=0, eps=1e-6, **kw):
    import paper_2604_09603_amd as pkg
    pkg.echo_store_latent(kv, weight, eps, pos, f, scale, layout, kv.shape[0], 512, 64, new, slots, pages, ps, **kw)


def _rows_ok(got, kv, weight, eps, pos, f, scale, layout):
    """Dims 0-511: the sum of squares has 14 additions and products of 2^-24 each (relative: all
    terms are positive), half of that in the root, 2^-22 for it, two products, the
    output's rounding 2^-8; without a weight, copies."""
    want = latent.latent_rows(kv, weight, eps, pos, f, scale, layout)
    c, o = f64(got[:, :512]), want[:, :512]
    if weight is None:
        assert np.array_equal(got[:, :512], kv[:, :512])
    else:
        tol = np.abs(o) * (2.0 ** -8 + (7 + 4 + 2) * 2.0 ** -24 * (1 + 2.0 ** -8)) + 2.0 ** -134
        assert np.all(np.abs(c - o) <= tol), np.abs(c - o).max()
    if f is None:
        assert np.array_equal(got[:, 512:], kv[:, 512:576])
    else:
        _rotated_ok(got[:, 512:], f64(kv[:, 512:576]), pos, f, scale, layout)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("lens,starts,ps,stride", [
    ([1], [0], 32, 576), ([1, 1, 1], [31, 32, 77], 32, 584), ([5, 100, 1, 40], [30, 61, 95, 0], 64, 576),
    ([700, 0, 3], [0, 9, 250], 256, 640), ([1] * 70, list(range(70)), 128, 2112)])
def test_store_matches_oracle(lens, starts, ps, stride, layout):
    import torch
    rng = np.random.default_rng(sum(lens))
    slots, npages = _slots_of(lens, starts, ps, rng)
    T = len(slots)
    wide = _bf(rng.standard_normal((T, stride)) * np.exp2(rng.integers(-6, 7, (T, 1))))
    kv, weight = wide[:, :576], _bf(1 + 0.1 * rng.standard_normal(512))
    pos = np.concatenate([np.arange(s, s + n) for s, n in zip(starts, lens)])
    f, scale = latent.frequencies(64, 10000.0, "bands", 40.0, 4096.0)
    pages = rng.integers(0, 1 << 16, (npages, ps, 576)).astype(np.uint16)
    _log(f"[store] T={T} page={ps} stride={stride} layout={layout}")
    kvd, pd, sd = _dev(wide)[:, :576], _dev(pages), _dev(slots)
    new = torch.zeros((T, 576), dtype=torch.bfloat16, device="cuda:0")
    args = (kvd, _dev(weight), _dev(pos, np.int32), _dev(f), scale, layout)
    status = _zeros(1)
    _store(*args, new=new, slots=sd, pages=pd, ps=ps, status=status)  # both at once
    _rows_ok(_bits(new), kv, weight, 1e-6, pos, f, float(np.float32(scale)), layout)
    want = pages.copy()
    want.reshape(-1, 576)[slots] = _bits(new)
    assert np.array_equal(_bits(pd), want) and int(status.item()) == 0
    alone, pd2 = torch.zeros_like(new), _dev(pages)
    _store(*args, new=alone)
    _store(*args, slots=sd, pages=pd2, ps=ps)
    assert torch.equal(alone.view(torch.int16), new.view(torch.int16))
    assert torch.equal(pd2.view(torch.int16), pd.view(torch.int16))


def test_rope_one_row_of_heads_far_apart():
    """The row stride of a tensor of one row says nothing, whatever its head stride."""
    import torch
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(5)
    far = 1 << 28                                   # (times 8 heads: 2^31)
    x = torch.empty(7 * far + 64, dtype=torch.bfloat16, device="cuda:0").as_strided((1, 8, 64), (1, far, 1))
    x.copy_(_dev(_bf(rng.standard_normal((1, 8, 64)))))
    near, want = x.contiguous(), torch.zeros((1, 8, 64), dtype=torch.bfloat16, device="cuda:0")
    f, s = latent.frequencies(64, 1e4)
    pos, f = _dev([4097], np.int32), _dev(f)
    pkg.echo_rope(near, want, None, None, pos, 1, 8, 0, 64, 0, f, s)
    pkg.echo_rope(x, x, None, None, pos, 1, 8, 0, 64, 0, f, s)
    assert torch.equal(x.contiguous().view(torch.int16), want.view(torch.int16))


def test_store_in_place():
    """Rows of kv themselves, where none moves; one row of a wider matrix."""
    import torch
    rng = np.random.default_rng(4)
    kv, weight = _bf(rng.standard_normal((3001, 640))), _bf(rng.standard_normal(512))
    pos, (f, s) = rng.integers(0, 5000, 3001), latent.frequencies(64, 1e4)
    args = (_dev(weight), _dev(pos, np.int32), _dev(f), s, 1)
    x = _dev(kv)[:, :576].contiguous()
    want = torch.zeros_like(x)
    _store(x, *args, new=want)
    _store(x, *args, new=x)
    assert torch.equal(x.view(torch.int16), want.view(torch.int16))
    one = _dev(kv)[:1]
    _store(one[:, :576], *args, new=one)
    assert torch.equal(one[0, :576].view(torch.int16), want[0].view(torch.int16))
    assert np.array_equal(_bits(one)[0, 576:], kv[0, 576:])


def test_store_without_norm_or_rotation():
    import torch
    rng = np.random.default_rng(1)
    kv, weight = _bf(rng.standard_normal((9, 576))), _bf(rng.standard_normal(512))
    pos, (f, s) = rng.integers(0, 500, 9), latent.frequencies(64, 1e4)
    for w, ff in [(None, None), (weight, None), (None, f)]:
        new = torch.zeros((9, 576), dtype=torch.bfloat16, device="cuda:0")
        _store(_dev(kv), None if w is None else _dev(w), None if ff is None else _dev(pos, np.int32),
               None if ff is None else _dev(ff), s, 0, new=new)
        _rows_ok(_bits(new), kv, w, 1e-6, pos, ff, s, 0)


def test_store_slots_and_rows_that_take_no_part():
    """Negative slots, slots past the pool, rows past the count; a row of zeros; eps 0."""
    import torch
    rng = np.random.default_rng(2)
    kv, weight, ps, npages = _bf(rng.standard_normal((40, 576))), _bf(np.ones(512)), 32, 3
    kv[4] = 0
    f, pos = latent.frequencies(64, 1e4)[0], rng.integers(0, 99, 40)
    pages = rng.integers(0, 1 << 16, (npages, ps, 576)).astype(np.uint16)
    slots = rng.permutation(npages * ps)[:40].astype(np.int64)
    slots[[3, 7, 20]] = -1, -5, np.iinfo(np.int64).min
    for beyond, n in [((), 40), ((npages * ps, 1 << 40), 40), ((), 11), ((), 0), ((), 41), ((), -1)]:
        sl = slots.copy()
        sl[30:30 + len(beyond)] = beyond
        pd, status = _dev(pages), _zeros(1)
        new = torch.full((40, 576), 3.0, dtype=torch.bfloat16, device="cuda:0")
        _store(_dev(kv), _dev(weight), _dev(pos, np.int32), _dev(f), 1.0, 1, new=new, slots=_dev(sl), pages=pd, ps=ps,
               row_count=_dev([n], np.int32), status=status)
        live = n if 0 <= n <= 40 else 0
        goes, bits = latent.slots_status(sl[:live], npages * ps)
        assert int(status.item()) == (bits if live == n else st.BAD_OFFSETS)
        got = _bits(new)
        _rows_ok(got[:live], kv[:live], weight, 1e-6, pos[:live], f, 1.0, 1)
        assert np.all(f64(got[live:]) == 3.0)
        want = pages.copy()
        want.reshape(-1, 576)[sl[:live][goes]] = got[:live][goes]
        assert np.array_equal(_bits(pd), want)
    new = torch.zeros((40, 576), dtype=torch.bfloat16, device="cuda:0")
    _store(_dev(kv[5:]), _dev(weight), _dev(pos[5:], np.int32), _dev(f), 1.0, 1, new=new[:35], eps=0.0)
    _rows_ok(_bits(new[:35]), kv[5:], weight, 0.0, pos[5:], f, 1.0, 1)


@pytest.mark.parametrize("ps", [32, 64])
@pytest.mark.parametrize("in_place", [False, True])
def test_commit_matches_oracle(ps, in_place):
    """Paths of 0 to 16 nodes over page borders; requests without slots, with missing pages, bad
    slots, lengths at the type's end."""
    rng = np.random.default_rng(ps)
    R, cap, depth = 40, 200, 16
    qo = np.concatenate([[0], np.cumsum(rng.integers(0, 6, R))]).astype(np.int32)
    plen = rng.integers(0, 100, R).astype(np.int32)
    alen = rng.integers(0, depth + 1, R).astype(np.int32)
    slots = rng.integers(0, cap, (R, depth)).astype(np.int32)
    max_pages = -(-(100 + depth + 1) // ps)
    npages = R * max_pages + 3
    bt = rng.permutation(npages)[:R * max_pages].reshape(R, max_pages).astype(np.int32)
    bt[3] = -1
    bt[5] = npages
    slots[7, 0], alen[7] = cap, 3
    slots[9, 1], alen[9] = -1, 2
    alen[11], alen[13] = -1, depth + 1
    plen[15], plen[17] = -1, 2 ** 31 - 1
    plen[19] = max_pages * ps  # past the table
    new = rng.integers(0, 1 << 16, (cap, 576)).astype(np.uint16)
    pages = rng.integers(0, 1 << 16, (npages, ps, 576)).astype(np.uint16)
    want, wl, ws = latent.commit_latent(qo, alen, slots, new, pages, bt, plen)
    import paper_2604_09603_amd as pkg
    pd, ld, status = _dev(pages), _dev(plen), _zeros(1)
    out = ld if in_place else _zeros(R)
    _log(f"[commit] page={ps} in_place={in_place}")
    pkg.echo_commit_latent(_dev(qo), _dev(alen), _dev(slots), depth, _dev(new), R, cap, 512, 64, pd, ps, _dev(bt), ld,
                           out, status=status)
    assert np.array_equal(_bits(pd), want) and np.array_equal(out.cpu().numpy(), wl)
    assert int(status.item()) == ws == st.BAD_OFFSETS


def test_writers_on_other_streams_and_in_graphs():
    """Two streams at once over buffers of their own; captured calls replayed with changed inputs."""
    import torch
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(31)
    T, ps, f = 90, 32, latent.frequencies(64, 1e4)[0]
    slots, npages = _slots_of([T], [7], ps, rng)
    weight, df, ds = _dev(_bf(rng.standard_normal(512))), _dev(f), _dev(slots)
    bt, qo = _dev(rng.permutation(npages).reshape(1, -1).astype(np.int32)), _dev([0, 5], np.int32)
    path = np.full((1, 4), -1, np.int32)
    path[0, :2] = 2, 4
    alen, path = _dev([2], np.int32), _dev(path)

    class Side:
        def __init__(self):
            self.kv, self.pos = torch.zeros((T, 576), dtype=torch.bfloat16, device="cuda:0"), _zeros(T)
            self.new, self.q = torch.zeros_like(self.kv), torch.zeros((T, 9, 64), dtype=torch.bfloat16, device="cuda:0")
            self.pages = torch.zeros((npages, ps, 576), dtype=torch.bfloat16, device="cuda:0")
            self.plen, self.len = _zeros(1) + 30, _zeros(1)

        def fill(self, seed):
            r = np.random.default_rng(seed)
            self.x, self.at = _bf(r.standard_normal((T, 576))), r.integers(0, 4000, T).astype(np.int32)
            self.heads = _bf(r.standard_normal((T, 9, 64)))
            for a, b in ((self.kv, self.x), (self.pos, self.at), (self.q, self.heads)):
                a.copy_(_dev(b))

        def calls(self, **kw):
            _rope(self.q, self.q, None, None, self.pos, df, 1.0, 0, **kw)
            _store(self.kv, weight, self.pos, df, 1.0, 0, new=self.new, slots=ds, pages=self.pages, ps=ps, **kw)
            pkg.echo_commit_latent(qo, alen, path, 4, self.new, 1, T, 512, 64, self.pages, ps, bt, self.plen, self.len, **kw)

        def check(self):
            _rotated_ok(_bits(self.q), f64(self.heads), self.at, f, 1.0, 0)
            new = _bits(self.new)
            _rows_ok(new, self.x, _bits(weight), 1e-6, self.at, f, 1.0, 0)
            want = np.zeros((npages * ps, 576), np.uint16)
            want[slots] = new
            want, wl, _ = latent.commit_latent([0, 5], [2], path.cpu().numpy(), new, want.reshape(npages, ps, 576),
                                               bt.cpu().numpy(), [30])
            assert np.array_equal(_bits(self.pages), want) and self.len.item() == wl[0] == 33

    sides, streams = [Side(), Side()], [torch.cuda.Stream(), torch.cuda.Stream()]
    for k, s in enumerate(sides):
        s.fill(k)
    torch.cuda.synchronize()
    for s, stream in zip(sides, streams):
        s.calls(stream=stream)
    torch.cuda.synchronize()
    for s in sides:
        s.check()
    s = sides[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.calls()
    for k in range(3):
        s.fill(10 + k)
        x = torch.randn(256, 256, device="cuda:0")
        (x @ x).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        s.check()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rows,hq,hk,rot,at,wide", [
    (5000, 3, 1, 16, 0, 16), (2100, 1, 0, 8, 8, 24), (4099, 2, 1, 24, 72, 96), (6001, 1, 1, 6, 0, 6), (2048, 1, 0, 2, 0, 2),
    (3000, 5, 3, 48, 4, 56), (2500, 1, 1, 40, 2, 42), (300, 20, 1, 24, 0, 24), (7, 64, 4, 120, 8, 128)])
def test_rope_many_short_rows_and_narrow_vectors(rows, hq, hk, rot, at, wide, layout):
    """Workgroups of several rows, the last of them partly past the rows that exist; parts that start or
    end 16, 8 or 4 bytes into a head."""
    import torch
    rng = np.random.default_rng(rows + rot)
    f, scale = latent.frequencies(rot, 1e4) if rot > 2 else (np.ones(1), 1.0)
    pos, n = rng.integers(0, 5000, rows), rows - 3
    x = [_bf(rng.standard_normal((rows, h, wide))) for h in (hq, hk)]
    _log(f"[rope] rows={rows} heads={hq}+{hk} rot={rot} at={at} of {wide} layout={layout}")
    d = [_dev(v) if v.size else None for v in x]
    y = [torch.full((rows, v.shape[1], rot), 7.0, dtype=torch.bfloat16, device="cuda:0") for v in d if v is not None]
    y += [None] * (2 - len(y))
    status = _zeros(1)
    views = [v if v is None else v[..., at:at + rot] for v in d]
    _rope(views[0], y[0], views[1], y[1], _dev(pos, np.int32), _dev(np.array(f)), scale, layout,
          row_count=_dev([n], np.int32), status=status)
    for v, out in zip(x, y):
        if out is None:
            continue
        got = _bits(out)
        _rotated_ok(got[:n], f64(v[:n, :, at:at + rot]), pos[:n], np.array(f), scale, layout)
        assert np.all(f64(got[n:]) == 7.0)
    assert int(status.item()) == 0
    for v, t in zip(x, views):  # in place
        if t is not None:
            _rope(t, t, None, None, _dev(pos, np.int32), _dev(np.array(f)), scale, layout)
    for v, t, out in zip(x, d, y):
        if t is not None:
            got = _bits(t)
            assert np.array_equal(got[:n, :, at:at + rot], _bits(out)[:n])
            assert np.array_equal(got[..., :at], v[..., :at]) and np.array_equal(got[..., at + rot:], v[..., at + rot:])
