"""The 8-bit paged cache where its calls can go wrong: limits, scales, page checks, long ranges, bad offsets.
Attention is compared with a plain form in 64 bits."""
import numpy as np
import pytest

from oracle import kvq8, status as st
from tests import gpu_common as gc
from tests.test_gpu_kvq8 import _dev, _log, _zeros

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    gc.require_gpu()


def _attn(q, kn, vn, fmt, cache, ps, bt, plen, qo, mask, hq, hkv, scale=128 ** -0.5):
    """The call on device tensors: out and lse (NaN where nothing was written) and the status."""
    import torch
    import paper_2604_09603_amd as pkg
    from paper_2604_09603_amd.step import _aligned_workspace
    R, cap = len(plen), q.shape[0]
    out = torch.full((cap, hq, 128), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    lse = torch.full((cap, hq), float("nan"), dtype=torch.float32, device="cuda:0")
    ws = _aligned_workspace(pkg.tree_verify_attn_paged_q8_workspace_size(R, cap, hq, hkv, bt.shape[1]), "cuda:0")
    ws.fill_(0xCD)
    status = _zeros(1)
    pkg.echo_tree_verify_attn_paged_q8(q, kn, vn, fmt, *cache, ps, bt, plen, qo, mask, mask.shape[1], R, cap,
                                       hq, hkv, 128, scale, out, lse, ws, status=status)
    torch.cuda.synchronize()
    return out, lse, int(status.item())


@pytest.mark.parametrize("tokens,slots,hq", [(4 << 20, 1, 8), ((4 << 20) - 63, 3, 128), ((1 << 31) - (1 << 20), 12, 64)])
def test_more_steps_than_a_call_takes(tokens, slots, hq):
    """2048 requests of millions of tokens over one shared page ask for more than 2^30 steps: nothing
    is computed, and the status says so.  A head's rows are those of one wave, of a gang of two and of a
    gang of four."""
    import torch
    _log(f"[attn q8] {tokens} tokens for 2048 requests of {slots} slots")
    R, hkv, ps = 2048, 8, 1 << 20
    assert R * hkv * (2 + -(-tokens // 64)) > 1 << 30
    cap = R * slots
    page = torch.zeros((1, hkv, ps, 128), dtype=torch.uint8, device="cuda:0")
    scale = torch.ones((1, hkv, ps // 32), dtype=torch.float32, device="cuda:0")
    bt = _zeros(R, -(-tokens // ps))
    plen = torch.full((R,), tokens, dtype=torch.int32, device="cuda:0")
    qo = torch.arange(R + 1, dtype=torch.int32, device="cuda:0") * slots
    kn = torch.zeros((cap, hkv, 128), dtype=torch.int16, device="cuda:0")
    q = torch.zeros((cap, hq, 128), dtype=torch.int16, device="cuda:0")
    mask = torch.ones((cap, 1), dtype=torch.int32, device="cuda:0")
    out, lse, status = _attn(q, kn, kn, kvq8.E4M3, (page, page, scale, scale), ps, bt, plen, qo, mask, hq, hkv)
    assert status == st.BAD_OFFSETS
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())


# ---- against a plain form in 64 bits ----------------------------------------

def _decode(pages, fmt):
    import torch
    return pages.view(torch.float8_e4m3fn if fmt == kvq8.E4M3 else torch.float8_e5m2).to(torch.float64)


def _plain(q, kn, vn, fmt, cache, ps, bt, plen, qo, mask, hq, hkv, scale):
    """Attention in 64 bits from its definition, request by request, on device tensors (q, kn and vn bf16).
    Returns out, lse and, for the bounds below, the weighted mean of |v - out| and of |v|, the
    largest sum of |q k| and the keys of a row; NaN for requests with lengths, offsets or pages that
    cannot be."""
    import torch
    R, G, cap = len(plen), hq // hkv, q.shape[0]
    n_pages = cache[0].shape[0]
    f64 = dict(dtype=torch.float64, device="cuda:0")
    out, dev, mabs = (torch.full((cap, hq, 128), float("nan"), **f64) for _ in range(3))
    lse, zabs, keys = (torch.full((cap, hq), float("nan"), **f64) for _ in range(3))
    table, lens, offs = bt.cpu().tolist(), plen.cpu().tolist(), qo.cpu().tolist()
    for r in range(R):
        a, b, P = offs[r], offs[r + 1], lens[r]
        need = -(-P // ps)
        if not (0 <= a <= b <= cap and 0 <= P and need <= bt.shape[1]):
            continue
        ids = table[r][:need]
        n = b - a
        if n == 0 or any(not 0 <= i < n_pages for i in ids):
            continue
        at = torch.tensor(ids, dtype=torch.int64, device="cuda:0")
        K, V = (torch.cat([(_decode(cache[i][at], fmt) * cache[2 + i][at].double().repeat_interleave(32, 2)[..., None]
                            ).transpose(0, 1).reshape(hkv, -1, 128)[:, :P], x[a:b].double().transpose(0, 1)], 1)
                for i, x in ((0, kn), (1, vn)))
        j = torch.arange(n, device="cuda:0")
        w = j >> 5
        bits = mask[a:b, w.clamp(max=mask.shape[1] - 1)].long() >> (j & 31) & 1
        see = torch.cat([torch.ones((n, P), dtype=torch.bool, device="cuda:0"), (bits > 0) & (w < mask.shape[1])], 1)
        Q = q[a:b].double().view(n, hkv, G, 128).permute(1, 0, 2, 3).reshape(hkv, n * G, 128)
        see = see[:, None, :].expand(n, G, P + n).reshape(1, n * G, P + n)
        # K's columns side by side: products of plain matrices, head by head
        z = torch.stack([Q[h] @ K[h].T.contiguous() for h in range(hkv)]).mul_(float(scale))
        za = torch.stack([Q[h].abs() @ K[h].abs().T.contiguous() for h in range(hkv)]).mul_(float(scale))
        z.masked_fill_(~see, -float("inf"))
        za.masked_fill_(~see, 0.0)
        m = z.amax(-1, keepdim=True).clamp(min=-1e300)
        p = (z - m).exp_()
        l = p.sum(-1, keepdim=True)
        p /= l.clamp(min=1e-300)
        o = torch.stack([p[h] @ V[h] for h in range(hkv)])
        ma = torch.stack([p[h] @ V[h].abs() for h in range(hkv)])
        # mean |v - o| <= the root of the mean square
        sq = torch.stack([p[h] @ (V[h] * V[h]) for h in range(hkv)])
        de = (sq - o * o).clamp_(min=0.0).sqrt_()
        back = lambda x: x.view(hkv, n, G, -1).permute(1, 0, 2, 3).reshape(n, hq, -1)  # noqa: E731
        out[a:b], dev[a:b], mabs[a:b] = back(o), back(de), back(ma)
        lse[a:b] = back(m + l.log())[..., 0]
        zabs[a:b], keys[a:b] = back(za.amax(-1, keepdim=True))[..., 0], float(P + n)
    return dict(out=out, lse=lse, dev=dev, mabs=mabs, zabs=zabs, keys=keys)


def _check(got, ref, chain, what=""):
    """Bounds per element, from the call's documented roundings; u = 2^-24 is half a step of fp32.
    * each weight is rounded to bf16 (2^-8 of it) and the sum is that of the rounded ones: 2^-8 /
      (1 - 2^-8) of the mean |v - o|;
    * a score: 129 products and sums and as many again for the factors, u each on sum |q k|; the exponential
      2^-22: a relative error of the weights, on the same mean;
    * fp32 sums: chain additions one after another (the keys of a wave's range and the merged parts),
      u each on the mean |v|; the log of the sum the same, and 2^-18 for the exponents of scales;
    * the output's rounding to bf16, 2^-8 of it."""
    import torch
    out, lse = got[0].double(), got[1].double()
    live = ~torch.isnan(ref["lse"])
    assert bool((torch.isnan(lse) == ~live).all()), f"{what}: rows written or not"
    assert bool((torch.isnan(out) == ~live[..., None]).all()), f"{what}: outputs written or not"
    u = 2.0 ** -24
    x = {n: t[live] for n, t in ref.items()}
    o, l = out[live], lse[live]
    dz = x["zabs"] * (2 * 129 * u)
    tol = x["dev"] * (2.0 ** -8 / (1 - 2.0 ** -8) + dz[:, None] + 2.0 ** -22) + x["mabs"] * (chain * u)
    tol = tol * (1 + 2.0 ** -7) + x["out"].abs() * 2.0 ** -8
    err = (o - x["out"]).abs()
    assert bool((err <= tol).all()), f"{what}: off by {float((err / tol.clamp(min=1e-300)).max()):.3f} of the bound"
    empty = torch.isneginf(x["lse"])
    assert bool((torch.isneginf(l) == empty).all()) and not bool(o[empty].any())
    f = ~empty
    tol = dz[f] + chain * u + 2.0 ** -18 + x["lse"][f].abs() * 2.0 ** -22
    err = (l[f] - x["lse"][f]).abs()
    assert bool((err <= tol).all()), f"{what}: lse off by {float((err / tol).max()):.3f} of the bound"


def _bf16(x):
    import torch
    return torch.as_tensor(np.asarray(x, np.float32)).to(torch.bfloat16).to("cuda:0")


def _chains(n, rng):
    """Masks of n slots that see themselves and some of those before."""
    W = max(1, -(-n // 32))
    m = np.zeros((n, W), np.uint32)
    for j in range(n):
        if j:
            m[j] = m[rng.integers(max(0, j - 5), j)]
        m[j, j >> 5] |= np.uint32(1 << (j & 31))
    return m


@pytest.mark.parametrize("fmt", [kvq8.E4M3, kvq8.E5M2])
def test_values_far_below_the_dominant_keys(fmt):
    """Half of the keys have all the weight and values of zero, the others 2^-57 of it and values near
    2^-62: rows whose sums are near 2^-115 where their units are split between waves."""
    import torch
    rng = np.random.default_rng(30)
    P, ps, hq, hkv = 4000, 64, 8, 2
    pages = -(-P // ps)
    kb = np.zeros((pages, hkv, ps, 128), np.uint8)
    vb = np.zeros_like(kb)
    kb[:, :, 1::2, 0] = kvq8.encode8(np.float64(-40.0), fmt)
    vb[:, :, 1::2] = kvq8.encode8(rng.choice([-0.25, 0.25, 0.5], vb[:, :, 1::2].shape), fmt)
    ks = np.ones((pages, hkv, ps // 32), np.float32)
    vs = np.full_like(ks, 2.0 ** -60)
    cache = [torch.from_numpy(a).to("cuda:0") for a in (kb, vb, ks, vs)]
    q = np.zeros((1, hq, 128))
    q[..., 0] = 1.0
    kn = np.zeros((1, hkv, 128))
    kn[..., 0] = -90.0
    args = (_bf16(q), _bf16(kn), _bf16(kn * 0), fmt, cache, ps, torch.arange(pages, dtype=torch.int32, device="cuda:0")[None],
            torch.tensor([P], dtype=torch.int32, device="cuda:0"), torch.tensor([0, 1], dtype=torch.int32, device="cuda:0"),
            torch.ones((1, 1), dtype=torch.int32, device="cuda:0"), hq, hkv, 1.0)
    ref = _plain(*args)
    top = float(ref["out"].abs().max())
    assert 2.0 ** -125 < top < 2.0 ** -114
    _log(f"[attn q8] outputs up to {top:.2g}, fmt={fmt}")
    got = _attn(*args)
    assert got[2] == 0
    _check(got, ref, 1000, "tiny sums")


@pytest.mark.parametrize("fmt", [kvq8.E4M3, kvq8.E5M2])
@pytest.mark.parametrize("k_exp,v_exps", [(-60, (-60,)), (60, (60,)), (0, (-60, 60)), (60, (-60, 0, 60)), (-3, (-1, 0, 1))])
def test_scales_at_both_ends(fmt, k_exp, v_exps):
    """K scales of 2^-60 and 2^60, V scales at either end and both in one row; in units that waves share
    and in others."""
    import torch
    rng = np.random.default_rng(31)
    hq, hkv, ps, lens, slots = 16, 2, 64, [3000, 40, 64, 500], [2, 1, 5, 9]
    need = [-(-n // ps) for n in lens]
    pages = sum(need)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(5)
    t = torch.float8_e4m3fn if fmt == kvq8.E4M3 else torch.float8_e5m2
    cache = [torch.randn((pages, hkv, ps, 128), generator=gen, device="cuda:0").mul_(16.0).to(t).view(torch.uint8)
             for _ in range(2)]
    cache.append(torch.full((pages, hkv, ps // 32), 2.0 ** k_exp, device="cuda:0"))
    cache.append(torch.from_numpy(np.exp2(rng.choice(v_exps, (pages, hkv, ps // 32))).astype(np.float32)).to("cuda:0"))
    bt = np.full((len(lens), max(need)), -1, np.int32)
    ids, at = rng.permutation(pages), 0
    for r, n in enumerate(need):
        bt[r, :n] = ids[at:at + n]
        at += n
    qo = np.concatenate([[0], np.cumsum(slots)]).astype(np.int32)
    cap = int(qo[-1])
    mask = np.concatenate([_chains(n, rng) for n in slots])
    q = _bf16(rng.standard_normal((cap, hq, 128)) * 2.0 ** (-k_exp - 4))
    kn = _bf16(rng.standard_normal((cap, hkv, 128)) * 2.0 ** (k_exp + 4))
    vn = _bf16(rng.standard_normal((cap, hkv, 128)) * 2.0 ** v_exps[-1])
    args = (q, kn, vn, fmt, cache, ps, _dev(bt), _dev(np.array(lens, np.int32)), _dev(qo), _dev(mask), hq, hkv)
    _log(f"[attn q8] K scale 2^{k_exp}, V scales 2^{v_exps}, fmt={fmt}")
    got = _attn(*args)
    assert got[2] == 0
    _check(got, _plain(*args, 128 ** -0.5), 1000, f"{k_exp} {v_exps}")


# ---- page checks --------------------------------------------------------------

def _pool(pages, hkv, ps, fmt, seed, spare=1):
    """Random pages and scales, with a page of memory behind them (as views): an id that is missed reads that."""
    import torch
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    t, gain = (torch.float8_e4m3fn, 1.0) if fmt == kvq8.E4M3 else (torch.float8_e5m2, 2.0 ** 7)
    n = pages + spare
    c = [torch.randn((n, hkv, ps, 128), generator=gen, device="cuda:0").mul_(50.0 * gain).to(t).view(torch.uint8)[:pages]
         for _ in range(2)]
    return c + [torch.exp2(torch.randint(-9, -5, (n, hkv, ps // 32), generator=gen, device="cuda:0").float()).div_(gain)[:pages]
                for _ in range(2)]


def _new(cap, hq, hkv, seed, q_scale=1.0):
    rng = np.random.default_rng(seed)
    return (_bf16(rng.standard_normal((cap, hq, 128)) * q_scale), _bf16(rng.standard_normal((cap, hkv, 128))),
            _bf16(rng.standard_normal((cap, hkv, 128))))


def _skip(ref, rows):
    for t in ref.values():
        t[rows] = float("nan")
    return ref


@pytest.mark.parametrize("width", [512, 513])
@pytest.mark.parametrize("at", [0, 63, 64, 127, 128, 255, 256, "last"])
def test_page_checks_of_long_requests(width, at):
    """An id past the pool at place `at` of a request's pages, for requests of 64 to 500 pages; the widest
    table that the attention's waves check themselves, and one that has a launch of its own."""
    rng = np.random.default_rng(40)
    ps, hq, hkv = 32, 4, 1
    need = [64, 65, 3, 128, 129, 256, 257, 500]
    lens = [ps * n - int(rng.integers(0, ps)) for n in need]
    slots = [1, 2, 1, 9, 1, 30, 2, 1]
    pages = 600
    cache = _pool(pages, hkv, ps, kvq8.E4M3, 41)
    table = rng.integers(0, pages, (len(need), width)).astype(np.int32)
    qo = np.concatenate([[0], np.cumsum(slots)]).astype(np.int32)
    q, kn, vn = _new(int(qo[-1]), hq, hkv, 42)
    mask = np.concatenate([_chains(n, rng) for n in slots])
    args = (q, kn, vn, kvq8.E4M3, cache, ps, _dev(table), _dev(np.array(lens, np.int32)), _dev(qo), _dev(mask), hq, hkv)
    ref = _plain(*args, 128 ** -0.5)
    for r, n in enumerate(need):
        place = n - 1 if at == "last" else at
        if place >= n:
            continue
        bad = table.copy()
        bad[r, place] = pages
        bad[r, n:] = -1  # (behind the request's pages: not looked at)
        _log(f"[attn q8] width {width}, request {r} of {n} pages, bad id at {place}")
        got = _attn(*args[:6], _dev(bad), *args[7:])
        assert got[2] == st.BAD_OFFSETS
        _check(got, _skip({k: t.clone() for k, t in ref.items()}, slice(int(qo[r]), int(qo[r + 1]))), 1000, f"request {r}")


def test_page_checks_of_later_requests_of_a_range():
    """2000 requests over the same 130 pages: a wave's range holds several of them, and some have a bad id
    at a place that each step of the check looks at.  (One request with a row for each, which sees the
    prefix and itself, is the same computation.)"""
    import torch
    rng = np.random.default_rng(43)
    R, ps, hq, hkv, n = 2000, 32, 2, 2, 130
    P = ps * n - 5
    cache = _pool(n, hkv, ps, kvq8.E4M3, 44)
    q, kn, vn = _new(R, hq, hkv, 45)
    order = rng.permutation(n).astype(np.int32)
    ident = np.zeros((R, -(-R // 32)), np.uint32)
    for r in range(R):
        ident[r, r >> 5] = 1 << (r & 31)
    i32 = dict(dtype=torch.int32, device="cuda:0")
    ref = _plain(q, kn, vn, kvq8.E4M3, cache, ps, _dev(order[None]), torch.tensor([P], **i32),
                 torch.tensor([0, R], **i32), _dev(ident), hq, hkv, 128 ** -0.5)
    table = np.tile(order, (R, 1))
    bad = rng.choice(R, 60, replace=False)
    for i, r in enumerate(bad):
        table[r, [0, 63, 64, 127, 128, 129][i % 6]] = n
    for width in (n, 513):
        wide = np.pad(table, ((0, 0), (0, width - n)), constant_values=-1)
        _log(f"[attn q8] 2000 requests, width {width}")
        got = _attn(q, kn, vn, kvq8.E4M3, cache, ps, _dev(wide), torch.full((R,), P, **i32),
                    torch.arange(R + 1, **i32), torch.ones((R, 1), **i32), hq, hkv)
        assert got[2] == st.BAD_OFFSETS
        _check(got, _skip({k: t.clone() for k, t in ref.items()}, torch.from_numpy(bad).to("cuda:0")), 10000, f"width {width}")


@pytest.mark.parametrize("R", [3, 700])
@pytest.mark.parametrize("width", [512, 513, 70000])
def test_pages_of_paused_requests(width, R):
    """Requests without slots and with up to 500 (70000) pages write nothing, but a bad id among their
    pages is reported, at any place; one behind them is not."""
    import torch
    rng = np.random.default_rng(46)
    ps, hq, hkv, pages = 32, 2, 1, 8
    cache = _pool(pages, hkv, ps, kvq8.E5M2, 47)
    n = 70000 if width == 70000 else 500
    lens = rng.integers(0, 99, R).astype(np.int32)
    slots = np.ones(R, np.int64)
    paused = R // 2
    slots[paused], lens[paused] = 0, n * ps - 3
    qo = np.concatenate([[0], np.cumsum(slots)]).astype(np.int32)
    q, kn, vn = _new(R - 1, hq, hkv, 48)
    table = torch.zeros((R, width), dtype=torch.int32, device="cuda:0")
    args = (q, kn, vn, kvq8.E5M2, cache, ps, table, _dev(lens), _dev(qo), _dev(np.ones((R - 1, 1), np.int32)), hq, hkv)
    ref = _plain(*args, 128 ** -0.5)
    for place in (None, 0, 1, 63, 64, 127, 128, 191, 256, n - 1, n):
        if place is not None and place < width:
            table[paused, place] = pages
        _log(f"[attn q8] {R} requests, width {width}, a paused one's bad id at {place}")
        got = _attn(*args)
        assert got[2] == (0 if place in (None, n) else st.BAD_OFFSETS)
        _check(got, ref, 100, f"place {place}")
        table[paused] = 0


@pytest.mark.parametrize("sm_scale", [1e-30, 1e-40])
def test_scores_that_vanish(sm_scale):
    """sm_scale times a K scale below the smallest number: every score is 0, and keys past a prefix or
    outside a row's mask still have no weight."""
    import torch
    rng = np.random.default_rng(50)
    ps, hq, hkv, lens, slots = 64, 8, 2, [1, 70, 1000, 64, 33], [2, 1, 3, 40, 1]
    need = [-(-n // ps) for n in lens]
    cache = _pool(sum(need), hkv, ps, kvq8.E4M3, 51)
    cache[2].fill_(2.0 ** -60)
    table, at = np.full((len(lens), max(need)), -1, np.int32), 0
    for r, n in enumerate(need):
        table[r, :n] = np.arange(at, at + n)
        at += n
    qo = np.concatenate([[0], np.cumsum(slots)]).astype(np.int32)
    q, kn, vn = _new(int(qo[-1]), hq, hkv, 52)
    W = max(-(-n // 32) for n in slots)
    mask = np.concatenate([np.pad(_chains(n, rng), ((0, 0), (0, W - max(1, -(-n // 32))))) for n in slots])
    args = (q, kn, vn, kvq8.E4M3, cache, ps, _dev(table), _dev(np.array(lens, np.int32)), _dev(qo), _dev(mask), hq, hkv,
            sm_scale)
    _log(f"[attn q8] sm_scale {sm_scale}")
    got = _attn(*args)
    assert got[2] == 0
    _check(got, _plain(*args), 1000, "vanishing scores")


# ---- commit -----------------------------------------------------------------

@pytest.mark.parametrize("below,accepted", [(5, 4), (1, 0), (0, 0), (4, 4), (3, 4)])
def test_commit_of_the_longest_requests(below, accepted):
    """A request of 2^31 - 1 - below tokens, all in one shared page of 2^20: the last token that a length of 31
    bits has is appended, a path that would go past it is not."""
    import torch
    import paper_2604_09603_amd as pkg
    ps, depth, top = 1 << 20, 4, (1 << 31) - 1
    P = top - below
    fits = 1 + accepted <= below
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(60)
    kn = torch.randn((depth + 1, 1, 128), generator=gen, device="cuda:0").abs_().add_(1.0).to(torch.bfloat16)
    page = [torch.zeros((1, 1, ps, 128), dtype=torch.uint8, device="cuda:0") for _ in range(2)]
    scale = [torch.ones((1, 1, ps // 32), device="cuda:0") for _ in range(2)]
    status, new = _zeros(1), _zeros(1)
    one = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    _log(f"[commit] {P} tokens and {1 + accepted} more")
    pkg.echo_commit_kv_q8(one([0, depth + 1]), one([accepted]), one([[1, 2, 3, 4]]), depth, kn, kn, 1, depth + 1, 1, 128,
                          kvq8.E4M3, *page, *scale, ps, _zeros(1, 2049), one([P]), new, status=status)
    assert int(status.item()) == (0 if fits else st.BAD_OFFSETS)
    assert int(new.item()) == (P + 1 + accepted if fits else P)
    want = sorted((P + i) % ps for i in range(1 + accepted)) if fits else []
    for t in page:
        assert t[0, 0].any(-1).nonzero()[:, 0].tolist() == want


def _one(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


@pytest.mark.parametrize("below,accepted", [(5, 4), (1, 0), (0, 0), (4, 4)])
def test_commit_of_the_longest_requests_in_bf16(below, accepted):
    """The same with the bfloat16 cache."""
    import torch
    import paper_2604_09603_amd as pkg
    ps, depth, top = 1 << 20, 4, (1 << 31) - 1
    P = top - below
    fits = 1 + accepted <= below
    kn = torch.ones((depth + 1, 1, 128), dtype=torch.bfloat16, device="cuda:0")
    page = [torch.zeros((1, ps, 1, 128), dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    status, length = _zeros(1), _one([P])
    _log(f"[commit] bf16, {P} tokens and {1 + accepted} more")
    pkg.echo_commit_kv(_one([0, depth + 1]), _one([accepted]), _one([[1, 2, 3, 4]]), depth, kn, kn, 1, depth + 1, 1,
                       *page, ps, _zeros(1, 2049), length, status=status)
    assert int(status.item()) == (0 if fits else st.BAD_OFFSETS)
    assert int(length.item()) == (P + 1 + accepted if fits else P)
    want = sorted((P + i) % ps for i in range(1 + accepted)) if fits else []
    for t in page:
        assert (t[0, :, 0] != 0).any(-1).nonzero()[:, 0].tolist() == want


# ---- block tables -------------------------------------------------------------

@pytest.mark.parametrize("max_rows", [60, 5000])
@pytest.mark.parametrize("rows", [[0, 7, 5, 30], [-1, 3, 9, 20], [4, 9, 20, "past"], [0, 0, 0, "past"], [-9, -9, -9, -9],
                                  ["past", 0, 1, 2], [0, 3, 9, "all"], [8, 8, 8, 8]])
def test_row_offsets_that_cannot_be(rows, max_rows):
    """Offsets that decrease, are negative or end past the slot map give no row a slot, and the status says
    so, with the slots in the tables' launch and in one of their own; the pages are dealt all the same."""
    from tests.test_gpu_kvq8 import _run_tables, _same_tables, _tables_case
    rng = np.random.default_rng(70)
    R, ps = 3, 32
    c = _tables_case(rng, R, 4, ps, 9, 20)
    c["ro"] = np.array([dict(past=max_rows + 1, all=max_rows).get(x, x) for x in rows], np.int32)
    _log(f"[tables] row offsets {rows}, {max_rows} rows")
    got = _run_tables(c, R, ps, max_rows, False)
    want = kvq8.build_block_tables(c["want"], ps, c["bt"], c["held"], c["stack"], c["free"], c["ro"], c["start"], max_rows)
    bad = "past" in rows or rows[0] < 0 or rows[2] < rows[1]
    assert bool(got["status"] & st.BAD_OFFSETS) == bad
    if bad:
        assert np.all(got["slot_map"] == -1)
    _same_tables(got, want)


def test_row_offsets_without_rows():
    """A slot map without rows: offsets that give requests rows end past it."""
    import torch
    import paper_2604_09603_amd as pkg
    one = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    lib = pkg.load()
    room = torch.full((4,), -7, dtype=torch.int64, device="cuda:0")
    for offs, want in (((0, 0), 0), ((0, 1), st.BAD_OFFSETS)):
        table, held, free, status = one(-1, -1), one(0), one(2), one(0)
        stack, lens, rows, start = one(5, 6), one(40), one(*offs), one(0)
        p = [t.data_ptr() for t in (lens, table, held, stack, free, rows, start, room, status)]
        _log(f"[tables] no rows, offsets {offs}")
        assert lib.echo_build_block_tables(p[0], 1, 32, p[1], 2, p[2], p[2], p[3], 2, p[4], p[4], p[5], p[6], 0, p[7], p[8],
                                           torch.cuda.current_stream().cuda_stream) == pkg.OK
        assert int(status.item()) == want and held.tolist() == [2] and table.tolist() == [6, 5]
        assert room.tolist() == [-7] * 4


# ---- long ranges ----------------------------------------------------------------

def _batch(lens, slots, hq, hkv, ps, fmt, seed, width=None, pool=None, head_scales=True):
    """Requests over random pages of a pool (which they share), heads whose scores are flat and others whose few
    largest have all the weight."""
    rng = np.random.default_rng(seed)
    need = [-(-int(n) // ps) for n in lens]
    pages = pool or max(sum(need), 1)
    cache = _pool(pages, hkv, ps, fmt, seed + 1)
    table = np.full((len(need), width or max(max(need), 1)), -1, np.int32)
    for r, n in enumerate(need):
        table[r, :n] = rng.integers(0, pages, n)
    qo = np.concatenate([[0], np.cumsum(slots)]).astype(np.int32)
    cap = int(qo[-1])
    scale = np.exp2(rng.integers(-1, 4, (cap, hq, 1))) if head_scales else 1.0
    q = _bf16(rng.standard_normal((cap, hq, 128)) * scale)
    kn, vn = (_bf16(rng.standard_normal((cap, hkv, 128))) for _ in range(2))
    W = max(1, -(-max(slots) // 32))
    mask = np.concatenate([np.zeros((0, W), np.uint32)] + [
        np.pad(_chains(n, rng), ((0, 0), (0, W - max(1, -(-n // 32))))) for n in slots if n])
    return [q, kn, vn, fmt, cache, ps, _dev(table), _dev(np.array(lens, np.int32)), _dev(qo), _dev(mask), hq, hkv]


@pytest.mark.parametrize("fmt", [kvq8.E4M3, kvq8.E5M2])
@pytest.mark.parametrize("R,slots,hq,kind", [(24, 1, 8, "waves alone"), (12, 5, 64, "gangs of two"), (6, 16, 64, "gangs of four"),
                                             (6, 9, 64, "gangs of four, one without rows"),
                                             (6, 20, 64, "gangs of four and waves alone"),
                                             (5, 36, 64, "two passes of gangs of four and one of two")])
def test_ranges_of_more_steps_than_a_table(R, slots, hq, kind, fmt):
    """Ranges of 40 to 60 steps: what a wave knows of its steps, 32 of them, is filled again on the way."""
    rng = np.random.default_rng(R)
    lens = rng.integers(30000, 32769, R)
    args = _batch(lens, [slots] * R, hq, 8, 64, fmt, 80 + slots, pool=700)
    _log(f"[attn q8] {kind}, fmt={fmt}")
    got = _attn(*args)
    assert got[2] == 0
    _check(got, _plain(*args, 128 ** -0.5), 5000, kind)


@pytest.mark.parametrize("slots,kind", [(5, "a gang of four"), (3, "a gang of two")])
def test_a_small_class_beside_a_large_one(slots, kind):
    """One request whose heads take gangs of four (or of two) beside 900 whose rows are one wave's: its class has
    two workgroups, and ranges of 45 (22) steps."""
    R = 901
    lens, n = np.full(R, 5600), [1] * R
    n[500] = slots
    lens[500] = 5600 * (1 if slots == 5 else 3)
    args = _batch(lens, n, 16, 1, 64, kvq8.E4M3, 90, pool=900)
    _log(f"[attn q8] {kind} beside 900 waves alone")
    got = _attn(*args)
    assert got[2] == 0
    _check(got, _plain(*args, 128 ** -0.5), 64 * 100, kind)


@pytest.mark.parametrize("width", [12, 600])
@pytest.mark.parametrize("slots,hq", [((1,), 16), ((3, 5), 64), ((9, 12, 20), 64), ((0, 1, 2, 4, 9, 17), 64)])
def test_many_short_requests_in_a_range(slots, hq, width):
    """1500 requests of 0 to 700 tokens: a range goes through several of them and its table is filled across
    their borders; every eighth has an id past the pool."""
    rng = np.random.default_rng(100 + width + len(slots))
    R, ps = 1500, 64
    lens = rng.integers(0, 701, R)
    lens[rng.random(R) < 0.1] = 0
    args = _batch(lens, rng.choice(slots, R).tolist(), hq, 8, ps, kvq8.E4M3, 101, width=width, pool=64)
    bad = args[6].cpu().numpy()
    for r in range(3, R, 8):
        if lens[r] > 0:
            bad[r, int(rng.integers(0, -(-lens[r] // ps)))] = 64
    args[6] = _dev(bad)
    _log(f"[attn q8] 1500 requests of {slots} slots, width {width}")
    got = _attn(*args)
    assert got[2] == st.BAD_OFFSETS
    _check(got, _plain(*args, 128 ** -0.5), 64 * 200, f"{slots}")


# ---- offsets --------------------------------------------------------------------

@pytest.mark.parametrize("width", [8, 600])
@pytest.mark.parametrize("flaw", ["negative", "past the rows", "decreasing", "all"])
def test_offsets_that_cannot_be(flaw, width):
    """Requests whose rows are not the call's are left out, beside healthy ones of every size of gang."""
    import torch
    slots = [1, 3, 6, 2, 1, 9, 4, 1]
    lens = [70, 200, 33, 0, 129, 300, 64, 5]
    args = _batch(lens, slots, 16, 1, 64, kvq8.E4M3, 110, width=width)
    qo = args[8].cpu().numpy().copy()
    cap = int(qo[-1])
    big = 2 ** 31 - 1
    if flaw == "negative":
        qo[0] = -1
    elif flaw == "past the rows":
        qo[-1] = cap + 1
    elif flaw == "decreasing":
        qo[3], qo[4] = big, qo[3]  # the third ends past the rows, the fourth begins there and ends before
    else:
        qo[0], qo[1], qo[4], qo[5], qo[-1] = -big - 1, 0, big, qo[4], -3
    args[8] = _dev(qo)
    _log(f"[attn q8] offsets {qo.tolist()}")
    got = _attn(*args)
    assert got[2] == st.BAD_OFFSETS
    ref = _plain(*args, 128 ** -0.5)
    assert 0 < int(torch.isnan(ref["lse"]).sum()) < cap * 16
    _check(got, ref, 500, flaw)


# ---- store ----------------------------------------------------------------------

@pytest.mark.parametrize("T", [1023, 1024, 1025, 2048, 2049])
def test_store_at_the_borders_of_rows_per_wave(T):
    """With two heads, up to 1024 rows have waves of their own and up to 2048 share one with another: runs
    that begin and end on either side of a wave's rows."""
    from tests.test_gpu_kvq8 import _empty_cache, _same_bytes, _slots_of, _store, _values
    rng = np.random.default_rng(T)
    hkv, ps = 2, 64
    lens, starts = [], []
    while sum(lens) < T:
        lens.append(min(int(rng.choice([1, 1, 2, 3, 33, 90])), T - sum(lens)))
        starts.append(int(rng.integers(0, 70)))
    slots, pages, _ = _slots_of(lens, starts, ps, rng)
    k, v = _values(rng, T, hkv, 128), _values(rng, T, hkv, 128)
    cache = _empty_cache(rng, pages, hkv, ps)
    dev = [_dev(a) for a in cache]
    _log(f"[store] {T} rows of two heads")
    _store(_dev(k), _dev(v), _dev(slots), kvq8.E4M3, dev, ps)
    *want, _ = kvq8.store_kv(k, v, slots, kvq8.E4M3, *cache)
    for i in range(2):
        _same_bytes(dev[i].cpu().numpy(), want[i], kvq8.E4M3, f"tensor {i}")
        assert np.array_equal(dev[2 + i].cpu().numpy(), want[2 + i])


@pytest.mark.parametrize("slots,hq", [(2, 4), (7, 16)])
def test_one_request_of_64_million_tokens(slots, hq):
    """A prefix that is one page of 2^20 tokens, 64 times: every wave fills its table again and again, and one
    unit is merged from all waves' sums.  The same as one page whose keys have 64 times the weight."""
    import torch
    ps, times = 1 << 20, 64
    cache = _pool(1, 1, ps, kvq8.E4M3, 120, spare=0)
    q, kn, vn = _new(slots, hq, 1, 121, q_scale=4.0)
    mask = _dev(_chains(slots, np.random.default_rng(122)))
    i32 = dict(dtype=torch.int32, device="cuda:0")
    _log(f"[attn q8] 2^26 tokens, {slots} slots")
    got = _attn(q, kn, vn, kvq8.E4M3, cache, ps, _zeros(1, times), torch.tensor([ps * times], **i32),
                torch.tensor([0, slots], **i32), mask, hq, 1)
    assert got[2] == 0
    K, V = (torch.cat([_decode(cache[i][0, 0], kvq8.E4M3) * cache[2 + i][0, 0].double().repeat_interleave(32)[:, None],
                       x[:, 0].double()]) for i, x in ((0, kn), (1, vn)))
    Q = q.double().view(slots * hq, 128) * 128 ** -0.5
    j = torch.arange(slots, device="cuda:0")
    see = (mask[:, j >> 5] >> (j & 31) & 1) > 0
    z = Q @ K.T.contiguous()
    za = Q.abs() @ K.abs().T.contiguous()
    z[:, :ps] += float(np.log(times))
    z[:, ps:].masked_fill_(~see.repeat_interleave(hq, 0), -float("inf"))
    m = z.amax(-1, keepdim=True)
    p = (z - m).exp_()
    l = p.sum(-1, keepdim=True)
    p /= l
    o = p @ V
    back = lambda x: x.view(slots, hq, -1)  # noqa: E731
    ref = dict(out=back(o), lse=back(m + l.log())[..., 0], dev=back(((p @ (V * V)) - o * o).clamp_(min=0.0).sqrt_()),
               mabs=back(p @ V.abs()), zabs=back(za.amax(-1, keepdim=True))[..., 0])
    # a wave has 2^20 steps of 64 keys among 2048 waves (512 gangs of four), and as many parts
    _check(got, ref, (1 << 20) * 64 // (2048 if slots * hq <= 32 else 512) * 1.15 + 2048, "2^26 tokens")


# ---- other calls that the documentation allows --------------------------------------

@pytest.mark.parametrize("slots,lens,hq,hkv", [([700, 1, 257], [1000, 64, 0], 4, 2), ([300], [31], 16, 1), ([1024, 33], [129, 2048], 8, 8)])
def test_prompt_chunks(slots, lens, hq, hkv):
    """Rows of a prompt over what is cached of it: a triangular mask of many words."""
    args = _batch(lens, [1] * len(lens), hq, hkv, 64, kvq8.E4M3, 130, head_scales=False)
    qo = np.concatenate([[0], np.cumsum(slots)]).astype(np.int32)
    cap = int(qo[-1])
    W = -(-max(slots) // 32)
    mask = np.zeros((cap, W), np.uint32)
    for r, n in enumerate(slots):
        for j in range(n):
            mask[qo[r] + j, :j >> 5] = 0xFFFFFFFF
            mask[qo[r] + j, j >> 5] = (2 << (j & 31)) - 1
    args[:3] = _new(cap, hq, hkv, 131, q_scale=2.0)
    args[8], args[9] = _dev(qo), _dev(mask)
    _log(f"[attn q8] prompt chunks of {slots} rows")
    got = _attn(*args)
    assert got[2] == 0
    _check(got, _plain(*args, 128 ** -0.5), 4000, "chunks")


def test_batch_of_paused_requests_only():
    """No request has slots: nothing is written, and their pages are checked all the same."""
    import torch
    args = _batch([70, 0, 200], [0, 0, 0], 8, 2, 64, kvq8.E4M3, 140)
    args[:3] = _new(5, 8, 2, 141)
    args[9] = _zeros(5, 1)
    for bad in (False, True):
        if bad:
            args[6][2, 1] = -1
        _log(f"[attn q8] paused requests only, bad={bad}")
        out, lse, status = _attn(*args)
        assert status == (st.BAD_OFFSETS if bad else 0)
        assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())


@pytest.mark.parametrize("rows", [2000, 5000])
def test_captured_tables_of_the_largest_batch(rows):
    """4095 requests, whose offsets take more shared memory than a kernel has by itself, captured and replayed on
    changing lengths with eager work between: every replay is the eager call."""
    import torch
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(150)
    R, most, ps, free = 4095, 3, 16, 9000
    held0 = rng.integers(0, most + 1, R).astype(np.int32)
    total = int(held0.sum()) + free
    perm = rng.permutation(total).astype(np.int32)
    bt0, at = np.full((R, most), -1, np.int32), 0
    for r in range(R):
        bt0[r, :held0[r]] = perm[at:at + held0[r]]
        at += int(held0[r])
    stack0 = np.full(total, -5, np.int32)
    stack0[:free] = perm[at:]
    init = [_dev(x) for x in (held0, bt0, stack0, np.array([free], np.int32))]
    held, bt, stack, nfree = (t.clone() for t in init)
    n = rng.multinomial(rows, np.ones(R) / R)
    ro = _dev(np.concatenate([[0], np.cumsum(n)]).astype(np.int32))
    want, start, status = _zeros(R), _zeros(R), _zeros(1)
    sm = torch.zeros(rows + 9, dtype=torch.int64, device="cuda:0")

    def call():
        pkg.echo_build_block_tables(want, R, ps, bt, held, held, stack, nfree, nfree, row_offsets=ro, row_start=start,
                                    slot_map=sm, status=status)

    def reset(seed):
        g = np.random.default_rng(seed)
        w = g.integers(0, most * ps + 1, R).astype(np.int32)
        want.copy_(_dev(w))
        start.copy_(_dev(np.maximum(0, w - n).astype(np.int32)))
        for t, u in zip((held, bt, stack, nfree), init):
            t.copy_(u)
        sm.fill_(-77)
        status.zero_()

    def fetch():
        torch.cuda.synchronize()
        return [t.cpu().numpy() for t in (held, bt, stack, nfree, sm, status)]

    eager = []
    for seed in range(3):
        reset(seed)
        call()
        eager.append(fetch())
    graph = torch.cuda.CUDAGraph()
    _log(f"[tables] 4095 requests captured, {rows} rows")
    with torch.cuda.graph(graph):
        call()
    for i in (1, 0, 2, 1):
        reset(i)
        graph.replay()
        for k, (a, b) in enumerate(zip(fetch(), eager[i])):
            assert np.array_equal(a, b), (i, k)
