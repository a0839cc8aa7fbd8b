"""GPU parity of the tree attention over the latent paged cache against the oracle, within the
roundings that the call documents."""
import numpy as np
import pytest

from oracle import latent, status as st
from tests import gpu_common as gc
from tests.test_gpu_latent import _bf, _bits, _dev, _log, _zeros

pytestmark = pytest.mark.gpu
NAN = 0x7FC0


@pytest.fixture(autouse=True)
def _need_gpu():
    gc.require_gpu()


def _tree(rng, n, W):
    """Random ancestor masks of n slots."""
    m = np.zeros((n, W), np.uint32)
    for j in range(n):
        if j:
            m[j] = m[rng.integers(max(0, j - 5), j)]
        m[j, j >> 5] |= np.uint32(1 << (j & 31))
    return m


def _case(rng, hq, slots, plens, ps, q_scale=1.0, spare=3, extra_pages=2, grow=None):
    """NaN wherever no request has a row.  grow: keys whose scores rise along the prefix."""
    R, cap = len(plens), sum(slots) + spare
    W = (max(slots) + 31) // 32 if max(slots) else 1
    qo = np.concatenate([[0], np.cumsum(slots)]).astype(np.int32)
    mask = np.zeros((cap, W), np.uint32)
    for r in range(R):
        mask[qo[r]:qo[r + 1]] = _tree(rng, slots[r], W)
    npg = [-(-p // ps) for p in plens]
    perm = rng.permutation(sum(npg) + extra_pages)
    bt = np.full((R, max(max(npg), 1)), -1, np.int32)
    pages = np.full((len(perm), ps, 576), NAN, np.uint16)
    at = 0
    q = rng.standard_normal((cap, hq, 576)) * q_scale
    for r in range(R):
        bt[r, :npg[r]] = perm[at:at + npg[r]]
        at += npg[r]
        x = rng.standard_normal((npg[r] * ps, 576))
        if grow is not None and plens[r] and slots[r]:
            x = x * 0.2 + np.linspace(0, grow, len(x))[:, None] * q[qo[r], 0] / 576
        x = _bf(x)
        x[plens[r]:] = NAN
        pages[bt[r, :npg[r]]] = x.reshape(npg[r], ps, 576)
    new = _bf(rng.standard_normal((cap, 576)))
    new[qo[-1]:] = NAN
    return dict(R=R, hq=hq, cap=cap, W=W, ps=ps, q=_bf(q), new=new, pages=pages, bt=bt, plen=np.array(plens, np.int32),
                qo=qo, mask=mask, scale=576 ** -0.5)


def _buffers(c):
    import torch
    import paper_2604_09603_amd as pkg
    from paper_2604_09603_amd.step import _aligned_workspace
    out = torch.full((c["cap"], c["hq"], 512), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    lse = torch.full((c["cap"], c["hq"]), float("nan"), dtype=torch.float32, device="cuda:0")
    ws = _aligned_workspace(pkg.tree_verify_attn_latent_workspace_size(c["R"], c["cap"], c["hq"], c["bt"].shape[1]),
                            "cuda:0")
    ws.fill_(0xFF)  # NaN everywhere
    return out, lse, ws, _zeros(1)


def _args(c, out, lse, ws, status):
    return (_dev(c["q"]), _dev(c["new"]), _dev(c["pages"]), c["ps"], _dev(c["bt"]), _dev(c["plen"]), _dev(c["qo"]),
            _dev(c["mask"]), c["W"], c["R"], c["cap"], c["hq"], 512, 64, c["scale"], out, lse, ws, status)


def _run(c):
    import torch
    import paper_2604_09603_amd as pkg
    out, lse, ws, status = _buffers(c)
    pkg.echo_tree_verify_attn_latent(*_args(c, out, lse, ws, status))
    torch.cuda.synchronize()
    return out.float().cpu().numpy(), lse.cpu().numpy(), int(status.item())


def _check(c, out, lse, status, want_status=0):
    """Error bounds, per element.  With w a row's weights, v its values, o its output:
    * the rounding of each w to bf16 (at most 2^-8 of it), sums of the rounded ones: the output
      moves by at most 2^-8 / (1 - 2^-8) of the mean |v - o|;
    * a score's fp32 error: 577 additions and products of 2^-24 each on sum |q k|, twice that for the
      exponent's products; an exponential's 2^-22: a relative error of w, on the same mean;
    * fp32 sums over n keys and up to 256 parts: a chain of n / 16 + 256 + 16 steps of 2^-24 of vmax;
    * the output's own rounding, 2^-8 of it."""
    ref = latent.tree_verify_attn_latent(c["q"], c["new"], c["pages"], c["bt"], c["plen"], c["qo"], c["mask"], c["hq"],
                                         c["scale"])
    assert status == ref["status"] == want_status
    nq = max(int(c["qo"][-1]), 0)
    live = ~np.isnan(ref["lse"])
    assert np.all(np.isnan(out[:nq]) == ~live[..., None]), "rows written or not"
    assert np.all(np.isnan(out[nq:])) and np.all(np.isnan(lse[nq:]))
    if not live.any():
        return
    o, l = out[:nq][live].astype(np.float64), lse[:nq][live].astype(np.float64)
    ro, rl = ref["out"][live], ref["lse"][live]
    dz = ref["zabs"][live][:, None] * (2 * 577 * 2.0 ** -24)
    keys = int(c["plen"].max()) + c["cap"]
    tol = (ref["dev"][live] * (2.0 ** -8 / (1 - 2.0 ** -8) + dz + 2.0 ** -22)
           + ref["vmax"][live][:, None] * (keys / 16 + 272) * 2.0 ** -24)
    tol = tol * (1 + 2.0 ** -7) + np.abs(ro) * 2.0 ** -8
    err = np.abs(o - ro)
    assert np.all(err <= tol), f"off by {np.nanmax(err / np.maximum(tol, 1e-300)):.3f} of the bound"
    empty = np.isneginf(rl)
    assert np.array_equal(np.isneginf(l), empty) and np.all(o[empty] == 0)
    f = ~empty
    assert np.all(np.abs(l[f] - rl[f]) <= dz[f, 0] + 2.0 ** -18 + np.abs(rl[f]) * 2.0 ** -22)


CASES = [
    # hq, slots, prefixes, page
    (1, [1], [0], 32), (1, [1], [1], 32), (1, [1, 1, 1], [31, 32, 33], 32), (16, [1], [640], 64),
    (16, [1, 1, 1], [31, 96, 200], 64), (16, [3, 1], [64, 65], 64), (128, [1], [300], 128), (128, [1, 3], [129, 40], 32),
    (64, [2, 1, 3], [96, 257, 0], 256), (20, [7, 0, 9], [130, 50, 1], 32), (5, [13, 26, 1], [33, 0, 777], 64),
    (32, [5, 4, 2, 1], [500, 33, 64, 1000], 32), (16, [33, 64, 65], [10, 0, 70], 32), (3, [100, 17], [31, 100], 64),
    (12, [6] * 9, [37 * i for i in range(9)], 32), (16, [8, 4], [1500, 900], 64), (127, [1, 2], [63, 31], 32),
    (129, [1, 1], [95, 1], 32), (300, [1], [70], 64)]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_matches_oracle(case):
    hq, slots, plens, ps = CASES[case]
    rng = np.random.default_rng(100 + case)
    _log(f"[latent attn] hq={hq} slots={slots} P={plens} page={ps}")
    c = _case(rng, hq, slots, plens, ps, q_scale=[1.0, 3.0][case % 2])
    _check(c, *_run(c))


@pytest.mark.parametrize("grow", [50.0, 3000.0, -3000.0, 40000.0])
@pytest.mark.parametrize("hq,slots,plens", [(16, [2, 1], [700, 900]), (64, [3, 1], [400, 65])])
def test_attention_rising_and_falling_scores(hq, slots, plens, grow):
    """References that are raised in many tiles, and parts whose weights vanish beside others."""
    rng = np.random.default_rng(int(abs(grow)) + hq)
    _log(f"[latent attn] grow={grow} hq={hq}")
    c = _case(rng, hq, slots, plens, 32, grow=grow)
    _check(c, *_run(c))


def test_attention_long_prefixes_are_cut():
    """Few requests over many workgroups: units of one range to many, equal and unequal."""
    for k, (hq, slots, plens) in enumerate([(2, [1], [20000]), (2, [1, 2], [5000, 9001]), (70, [1], [4000]),
                                            (1, [1] * 5, [3000, 0, 31, 8000, 1])]):
        _log(f"[latent attn] cut hq={hq} P={plens}")
        c = _case(np.random.default_rng(k), hq, slots, plens, 64)
        _check(c, *_run(c))


def test_attention_masks():
    """Rows that see nothing, one key, or another row's node; mask words that stop short."""
    rng = np.random.default_rng(8)
    c = _case(rng, 24, [5, 40, 3], [0, 0, 64], 32)
    c["mask"][0] = 0                      # sees nothing
    c["mask"][1] = [0b10000, 0]           # a later node only
    c["mask"][2] = 0xFFFFFFFF             # bits past the last slot
    c["mask"][5:45, 1] = 0                # nodes 32 .. see nothing of their own tile
    c["mask"][45] = 0                     # the prefix alone
    _check(c, *_run(c))
    c = _case(rng, 8, [40], [3], 32)      # one word for 40 slots: nodes past 31 are not seen
    c["mask"], c["W"] = np.ascontiguousarray(c["mask"][:, :1]), 1
    _check(c, *_run(c))


def test_attention_skips_bad_requests():
    rng = np.random.default_rng(9)
    hq, ps = 16, 32
    plens = [100, 200, 64, 130, 40, 90]
    for bad in ("low", "high", "late", "length", "negative", "none"):
        c = _case(rng, hq, [3, 9, 0, 2, 1, 4], plens, ps)
        if bad == "low":
            c["bt"][1, 0] = -1
        elif bad == "high":
            c["bt"][1, 1] = c["pages"].shape[0]
        elif bad == "late":
            c["bt"][1, 6] = 1 << 30
        elif bad == "length":
            c["plen"][1] = c["bt"].shape[1] * ps + 1
        elif bad == "negative":
            c["plen"][1] = -5
        else:
            c["bt"][2, :] = -7            # a request without slots: not looked at
        _log(f"[latent attn] bad request: {bad}")
        _check(c, *_run(c), 0 if bad == "none" else st.BAD_OFFSETS)


def test_attention_bad_offsets():
    rng = np.random.default_rng(10)
    c = _case(rng, 16, [3, 2, 4], [40, 50, 60], 32)
    c["qo"] = np.array([0, 3, 2, 9], np.int32)      # decreasing for request 1
    ref_qo = c["qo"].copy()
    out, lse, status = _run(c)
    assert status == st.BAD_OFFSETS and np.all(np.isfinite(lse[:3]))
    c["qo"] = np.array([0, 3, 5, c["cap"] + 1], np.int32)
    out, lse, status = _run(c)
    assert status == st.BAD_OFFSETS and np.all(np.isfinite(lse[:5])) and np.all(np.isnan(lse[5:]))
    c["qo"] = np.array([-1, 3, 5, 9], np.int32)
    out, lse, status = _run(c)
    assert status == st.BAD_OFFSETS and np.all(np.isnan(lse[:3])) and np.all(np.isfinite(lse[3:9]))
    assert ref_qo[1] == 3


def test_attention_many_requests():
    """More requests than workgroups, and than a workgroup has threads; most without slots."""
    rng = np.random.default_rng(11)
    for R, some in ((300, 1.0), (2000, 0.1)):
        slots = (rng.random(R) < some).astype(int) * rng.integers(1, 3, R)
        slots[0] = 0
        plens = rng.integers(0, 70, R)
        _log(f"[latent attn] R={R}")
        c = _case(rng, 2, slots.tolist(), plens.tolist(), 32)
        _check(c, *_run(c))


def test_attention_wide_block_tables():
    """Tables past the width that the main kernel checks by itself."""
    rng = np.random.default_rng(12)
    for bad in (False, True):
        c = _case(rng, 4, [2, 1, 1], [90, 32 * 700, 64], 32)
        assert c["bt"].shape[1] == 700
        wide = np.full((3, 1200), -1, np.int32)
        wide[:, :700] = c["bt"]
        c["bt"] = wide
        if bad:
            c["bt"][1, 650] = -1
        _check(c, *_run(c), st.BAD_OFFSETS if bad else 0)


def test_attention_cache_beyond_four_gigabytes():
    """Pages whose byte offsets pass 32 bits."""
    import torch
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(13)
    c = _case(rng, 16, [2, 1], [100, 60], 64, extra_pages=0)
    small = _run(c)
    shift = 70000                                   # 70000 pages of 73728 bytes: 5.2 GB
    pages = torch.empty((shift + c["pages"].shape[0], 64, 576), dtype=torch.bfloat16, device="cuda:0")
    pages[shift:] = _dev(c["pages"])
    out, lse, ws, status = _buffers(c)
    a = list(_args(c, out, lse, ws, status))
    a[2], a[4] = pages, _dev(np.where(c["bt"] >= 0, c["bt"] + shift, -1).astype(np.int32))
    pkg.echo_tree_verify_attn_latent(*a)
    assert np.array_equal(out.float().cpu().numpy(), small[0], equal_nan=True)
    assert np.array_equal(lse.cpu().numpy(), small[1], equal_nan=True)


def test_attention_captured_and_on_other_streams():
    """Replays of a captured call over changed lengths, with eager work between them; two streams
    with workspaces of their own."""
    import torch
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(14)
    c = _case(rng, 16, [4, 1, 7], [300, 900, 64], 64)
    out, lse, ws, status = _buffers(c)
    a = _args(c, out, lse, ws, status)
    pkg.echo_tree_verify_attn_latent(*a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.echo_tree_verify_attn_latent(*a)
    lens = [c["plen"].copy(), np.array([1, 0, 33], np.int32), np.array([290, 512, 0], np.int32), c["plen"].copy()]
    for plen in lens:
        a[5].copy_(torch.from_numpy(plen))
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        x = torch.randn(256, 256, device="cuda:0")
        (x @ x).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        _check(dict(c, plen=plen), out.float().cpu().numpy(), lse.cpu().numpy(), int(status.item()))
    two = [_case(rng, 16, [2, 3], [2000, 100], 64), _case(rng, 64, [1, 1], [700, 1200], 64)]
    bufs = [_buffers(c) for c in two]
    args = [_args(c, *b) for c, b in zip(two, bufs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s, x in zip(streams, args):
            pkg.echo_tree_verify_attn_latent(*x, stream=s)
    torch.cuda.synchronize()
    for c, b in zip(two, bufs):
        _check(c, b[0].float().cpu().numpy(), b[1].cpu().numpy(), int(b[3].item()))


def test_attention_is_deterministic_and_takes_no_lse():
    import torch
    import paper_2604_09603_amd as pkg
    rng = np.random.default_rng(15)
    c = _case(rng, 48, [3, 5, 1], [1500, 40, 3000], 128)
    out, lse, ws, status = _buffers(c)
    a = list(_args(c, out, lse, ws, status))
    pkg.echo_tree_verify_attn_latent(*a)
    first = _bits(out)
    for _ in range(3):
        out.fill_(float("nan"))
        ws.fill_(0xFF)
        pkg.echo_tree_verify_attn_latent(*a)
        assert np.array_equal(_bits(out), first)
    a[16] = None
    out.fill_(float("nan"))
    pkg.echo_tree_verify_attn_latent(*a)
    assert np.array_equal(_bits(out), first)
    torch.cuda.synchronize()


@pytest.mark.parametrize("hq,slots", [(1, 1), (40, 2)])
def test_attention_ranges_of_many_tiles(hq, slots):
    """More tiles to a workgroup than it keeps addresses of; requests that share pages."""
    rng = np.random.default_rng(16 + hq)
    R, ps = 64, 64
    c = _case(rng, hq, [slots] * R, [ps] * R, ps)
    c["plen"] = rng.integers(8900, 9500, R).astype(np.int32)
    full = np.flatnonzero(~np.any(c["pages"].reshape(len(c["pages"]), -1) == NAN, 1))
    c["bt"] = full[rng.integers(0, len(full), (R, 149))].astype(np.int32)
    _log(f"[latent attn] many tiles hq={hq}")
    out, lse, status = _run(c)
    assert status == 0 and np.all(np.isfinite(lse[:R * slots]))
    for r in (0, 1, 20, 41, 63):  # (each alone in the oracle)
        mine = slice(r * slots, (r + 1) * slots)
        one = dict(c, R=1, cap=slots, qo=np.array([0, slots], np.int32), **{k: c[k][mine] for k in ("q", "new", "mask")},
                   **{k: c[k][r:r + 1] for k in ("bt", "plen")})
        _check(one, out[mine], lse[mine], status)


def _among(c, rng, fillers=40, tokens=6000):
    """The requests of c with others behind them whose work makes the units as large as they get: the
    outputs and the status of c's own."""
    hq, ps, nq, W = c["hq"], c["ps"], max(int(c["qo"][-1]), 0), c["W"]
    n = -(-128 // hq)
    assert n <= 32 * W and int(c["qo"][-1]) <= c["cap"] and 2 * tokens // 32 * fillers > 2 * 6144
    cap = nq + n * fillers + 2
    fill = dict(q=_bf(rng.standard_normal((cap - nq, hq, 576))), new=_bf(rng.standard_normal((cap - nq, 576))),
                mask=np.zeros((cap - nq, W), np.uint32))
    fill["mask"][:, 0] = 1
    own = len(c["pages"])
    pages = np.concatenate([c["pages"], _bf(rng.standard_normal((64, ps, 576)))])
    bt = np.full((c["R"] + fillers, max(c["bt"].shape[1], -(-tokens // ps))), -1, np.int32)
    bt[:c["R"], :c["bt"].shape[1]] = c["bt"]
    bt[c["R"]:] = own + rng.integers(0, 64, (fillers, bt.shape[1]))
    big = dict(c, R=c["R"] + fillers, cap=cap, pages=pages, bt=bt, plen=np.concatenate([c["plen"], np.full(fillers, tokens, np.int32)]),
               qo=np.concatenate([c["qo"], nq + n * np.arange(1, fillers + 1)]).astype(np.int32),
               **{k: np.concatenate([c[k][:nq], v]) for k, v in fill.items()})
    big["bt"][:c["R"]] = np.where(big["bt"][:c["R"]] == own, len(pages), big["bt"][:c["R"]])  # (past the pool as before)
    out, lse, status = _run(big)
    assert np.all(np.isfinite(lse[nq:nq + n * fillers]))
    mine = [np.full((c["cap"],) + x.shape[1:], np.nan, np.float32) for x in (out, lse)]
    for a, b in zip(mine, (out, lse)):
        a[:nq] = b[:nq]
    return mine[0], mine[1], status


@pytest.mark.parametrize("case", [k for k, (hq, slots, _, _) in enumerate(CASES) if hq * max(slots) > 64])
def test_attention_large_units_match_oracle(case):
    hq, slots, plens, ps = CASES[case]
    rng = np.random.default_rng(200 + case)
    _log(f"[latent attn] large units hq={hq} slots={slots} P={plens} page={ps}")
    c = _case(rng, hq, slots, plens, ps, q_scale=[1.0, 3.0][case % 2])
    if hq * 32 * c["W"] < 128:  # (mask words for the others' slots)
        c["mask"], c["W"] = np.pad(c["mask"], ((0, 0), (0, -(-128 // hq // 32)))), c["W"] + -(-128 // hq // 32)
    _check(c, *_among(c, rng))


@pytest.mark.parametrize("grow", [50.0, 3000.0, -3000.0, 40000.0])
def test_attention_large_units_rising_and_falling_scores(grow):
    rng = np.random.default_rng(int(abs(grow)))
    c = _case(rng, 64, [3, 2], [700, 65], 32, grow=grow)
    _log(f"[latent attn] large units grow={grow}")
    _check(c, *_among(c, rng))


def test_attention_large_units_masks_and_bad_requests():
    rng = np.random.default_rng(17)
    c = _case(rng, 24, [5, 40, 4], [0, 0, 64], 32)
    c["mask"][0] = 0
    c["mask"][1] = [0b10000, 0]
    c["mask"][2] = 0xFFFFFFFF
    c["mask"][5:45, 1] = 0
    c["mask"][45] = 0
    _check(c, *_among(c, rng))
    for bad in ("low", "high", "length"):
        c = _case(rng, 16, [5, 9, 0, 7], [100, 200, 64, 130], 32)
        if bad == "low":
            c["bt"][1, 0] = -1
        elif bad == "high":
            c["bt"][1, 6] = c["pages"].shape[0]
        else:
            c["plen"][1] = -5
        _log(f"[latent attn] large units, bad request: {bad}")
        _check(c, *_among(c, rng), st.BAD_OFFSETS)


def _same_page(plens, max_pages, ps=1 << 20):
    """Requests whose block tables name one page of equal rows over and over."""
    import torch
    rng = np.random.default_rng(18)
    R, row = len(plens), _bf(rng.standard_normal(576))
    c = dict(R=R, hq=1, cap=R, W=1, ps=ps, q=np.zeros((R, 1, 576), np.uint16), new=np.tile(row, (R, 1)),
             bt=np.zeros((R, max_pages), np.int32), plen=np.array(plens, np.int32), qo=np.arange(R + 1, dtype=np.int32),
             mask=np.ones((R, 1), np.uint32), scale=0.05, pages=np.zeros((1, 1, 576), np.uint16))
    out, lse, ws, status = _buffers(c)
    a = list(_args(c, out, lse, ws, status))
    a[2] = torch.empty((1, ps, 576), dtype=torch.bfloat16, device="cuda:0")
    a[2][:] = _dev(row)
    return row, a, out, lse, status


def test_attention_very_long_prefix():
    """2^28 keys of equal rows and scores.  A workgroup's chain of sums is 2^16 steps of 16 keys, of O and of the
    weights' sum: 2^-24 each, and the output's rounding; the sums of whole numbers below 2^24 are
    exact, a part's, and a merge of 256 of them is off by 2^-24 each."""
    import paper_2604_09603_amd as pkg
    row, a, out, lse, status = _same_page([1 << 28], 257)
    _log("[latent attn] 2^28 keys")
    pkg.echo_tree_verify_attn_latent(*a)
    v, o = latent.bf16_to_f64(row[:512]), out.float().cpu().numpy()[0, 0].astype(np.float64)
    assert int(status.item()) == 0
    assert np.all(np.abs(o - v) <= np.abs(v) * (2 * 2.0 ** 16 * 2.0 ** -24 + 2.0 ** -8) * (1 + 2.0 ** -7))
    assert abs(float(lse.item()) - np.log(2.0 ** 28 + 1)) <= 256 * 2.0 ** -24 + 2.0 ** -18


def test_attention_refuses_more_work_than_it_counts():
    """16 requests of 2^31 keys: nothing is computed."""
    import torch
    import paper_2604_09603_amd as pkg
    n = 2047 << 20
    _, a, out, lse, status = _same_page([n] * 16, 2047)
    _log("[latent attn] too much work")
    pkg.echo_tree_verify_attn_latent(*a)
    assert int(status.item()) == st.BAD_OFFSETS
    assert torch.all(torch.isnan(out)) and torch.all(torch.isnan(lse))


@pytest.mark.parametrize("hq,slots", [(100, 3), (128, 2)])
def test_attention_units_of_a_request_side_by_side(hq, slots):
    """Long ranges that start in one unit of a request and hold the start of its next: taken out of order."""
    rng = np.random.default_rng(19 + hq)
    R, ps = 30, 64
    c = _case(rng, hq, [slots] * R, [ps] * R, ps)
    c["plen"] = rng.integers(2900, 3900, R).astype(np.int32)
    full = np.flatnonzero(~np.any(c["pages"].reshape(len(c["pages"]), -1) == NAN, 1))
    c["bt"] = full[rng.integers(0, len(full), (R, 61))].astype(np.int32)
    bad = 11                                            # found bad again when its first unit's end is done last
    c["bt"][bad, 30] = -1
    _log(f"[latent attn] side by side hq={hq}")
    out, lse, status = _run(c)
    assert status == st.BAD_OFFSETS
    live = np.ones(R * slots, bool)
    live[bad * slots:(bad + 1) * slots] = False
    assert np.all(np.isfinite(lse[:R * slots]) == live[:, None]) and np.all(np.isnan(out[:R * slots][~live]))
    for r in (0, 10, 12, 29):  # (each alone in the oracle)
        mine = slice(r * slots, (r + 1) * slots)
        one = dict(c, R=1, cap=slots, qo=np.array([0, slots], np.int32), **{k: c[k][mine] for k in ("q", "new", "mask")},
                   **{k: c[k][r:r + 1] for k in ("bt", "plen")})
        _check(one, out[mine], lse[mine], 0)


def _check_units_of_32(c, unit, out, lse, status):
    """Bounds of the last rows of each request, past whole units of `unit`: 32 at most, whose weights are taken in
    two bfloat16 numbers.  With w a row's weights, v its values, o its output:
    * w less its rounding to bf16 (2^-8 of it) is rounded to bf16 again, 2^-16 of w is left: 2^-16 of the mean
      |v|, which is at most the mean |v - o| and |o|;
    * a score's and an exponential's error and the output's own rounding as in _check;
    * fp32 sums: O's chain of two steps per 16 keys, the weights' of four per 32, each and a merge's 272 off by
      2^-24 a step."""
    ref = latent.tree_verify_attn_latent(c["q"], c["new"], c["pages"], c["bt"], c["plen"], c["qo"], c["mask"], c["hq"],
                                         c["scale"])
    assert status == ref["status"] == 0
    rows = np.concatenate([np.arange(a * c["hq"] + (b - a) * c["hq"] // unit * unit, b * c["hq"])
                           for a, b in zip(c["qo"], c["qo"][1:])])
    assert max((b - a) * c["hq"] % unit for a, b in zip(c["qo"], c["qo"][1:])) <= 32 and len(rows)
    o, ro, dev = (x.reshape(-1, 512)[rows].astype(np.float64) for x in (out, ref["out"], ref["dev"]))
    zabs, vmax, l, rl = (x.reshape(-1, 1)[rows] for x in (ref["zabs"], ref["vmax"], lse, ref["lse"]))
    keys = int(c["plen"].max()) + c["cap"]
    tol = ((dev + np.abs(ro)) * 2.0 ** -16 + dev * (zabs * (2 * 577 * 2.0 ** -24) + 2.0 ** -22)
           + vmax * 2 * (keys / 8 + 272) * 2.0 ** -24)
    tol = tol * (1 + 2.0 ** -7) + np.abs(ro) * 2.0 ** -8
    err = np.abs(o - ro)
    assert np.all(err <= tol), f"off by {(err / np.maximum(tol, 1e-300)).max():.3f} of the bound"
    assert np.array_equal(np.isneginf(l), np.isneginf(rl)) and np.all(o[np.isneginf(rl[:, 0])] == 0)


@pytest.mark.parametrize("hq,slots,plens", [
    (16, [1, 2, 1, 2], [1, 0, 5, 40]), (1, [1, 30, 3], [2, 0, 33]), (32, [1, 1], [3, 129]), (5, [6, 1], [31, 700]),
    (80, [1, 2], [4, 100]), (20, [1], [5000])])
def test_attention_units_of_32_rows_keep_their_weights(hq, slots, plens):
    """Cut and whole.  Small scores, whose fp32 error would hide a weight's rounding; rows of few keys, in whose
    outputs each would show."""
    rng = np.random.default_rng(21 + hq)
    _log(f"[latent attn] units of 32 hq={hq} P={plens}")
    c = _case(rng, hq, slots, plens, 32, q_scale=0.2)
    _check_units_of_32(c, 64, *_run(c))


@pytest.mark.parametrize("hq,slots,plens", [(16, [1, 2, 9], [3, 40, 700]), (32, [1, 5], [9, 300])])
def test_attention_units_of_32_rows_among_large_ones(hq, slots, plens):
    """Behind or beside units of 128 rows."""
    rng = np.random.default_rng(23 + hq)
    _log(f"[latent attn] units of 32 among large ones hq={hq} P={plens}")
    c = _case(rng, hq, slots, plens, 32, q_scale=0.2)
    _check_units_of_32(c, 128, *_among(c, rng))


@pytest.mark.parametrize("grow", [50.0, 3000.0, -3000.0, 40000.0])
def test_attention_units_of_32_rows_rising_and_falling_scores(grow):
    """References that are raised in many tiles, of the rows and of their second tile alike."""
    rng = np.random.default_rng(int(abs(grow)))
    _log(f"[latent attn] units of 32 grow={grow}")
    c = _case(rng, 16, [2, 1, 1], [700, 900, 33], 32, grow=grow)
    _check_units_of_32(c, 64, *_run(c))


@pytest.mark.parametrize("qo", [[0, 3, 2, 9], [5, 2, 9, 9], [0, 5, 3, 3], [0, 3, 5, 13], [-1, 3, 5, 9], [0, 3, 1 << 30, 9]])
def test_attention_values_beside_bad_offsets(qo):
    """Each well-formed request against the oracle with it alone; slots of no such request are left as they were, a
    slot of two holds either's output."""
    rng = np.random.default_rng(25)
    c = _case(rng, 16, [3, 2, 4], [40, 50, 60], 32)
    assert c["cap"] == 12
    c["qo"] = np.array(qo, np.int32)
    _log(f"[latent attn] offsets {qo}")
    out, lse, status = _run(c)
    assert status == st.BAD_OFFSETS
    own = [np.arange(a, b) if 0 <= a <= b <= 12 else np.arange(0) for a, b in zip(qo, qo[1:])]
    owners = np.bincount(np.concatenate(own).astype(int), minlength=12)
    assert np.all(np.isnan(out[owners == 0])) and np.all(np.isnan(lse[owners == 0]))
    for r, mine in enumerate(own):
        if len(mine) == 0:
            continue
        one = dict(c, R=1, cap=len(mine), qo=np.array([0, len(mine)], np.int32),
                   **{k: c[k][mine] for k in ("q", "new", "mask")}, **{k: c[k][r:r + 1] for k in ("bt", "plen")})
        o, l = out[mine], lse[mine]
        if np.any(owners[mine] > 1):  # (of which the oracle says what it may be)
            ref = latent.tree_verify_attn_latent(*(one[k] for k in ("q", "new", "pages", "bt", "plen", "qo", "mask",
                                                                    "hq", "scale")))
            o[owners[mine] > 1], l[owners[mine] > 1] = ref["out"][owners[mine] > 1], ref["lse"][owners[mine] > 1]
        _check(one, o, l, 0)
