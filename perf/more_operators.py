"""Latent attention's work, and rotary positions, at the sizes a serving engine gives them.

An engine whose model keeps one latent vector per token (512 normalised dims that serve
as keys and values of every head, and 64 rotated dims that only the scores see) rotates
its queries (``rope``), normalises and rotates the projection's rows on their way into
the paged cache or beside a draft tree (``store``), verifies trees or decodes single
tokens over the cache in every layer (``attn``), and appends the accepted rows
(``commit``).  Models with ordinary heads rotate queries and keys with the same call.

``run`` computes an operator in its plain form, or with ``own`` through the library's
calls.  Sizes are those of the workload presets with a latent cache in place of theirs;
what ``draw`` gives lies in the ranges that they span, odd and ragged sizes among them.
"""
import math

import numpy as np
import torch

own = False

LATENT, ROPE = 512, 64
ROW = LATENT + ROPE
DEV = "cuda:0"
MAX_DEPTH = 16
EPS = 1e-6

# What a drawn case may cost at most: the listed cases' largest.
MAX_CACHE_BYTES = 7e8
MAX_FLOPS = 7e11
MAX_ROPE_BYTES = 8e8
MAX_STORE_ROWS = 40000


def _case(kind, name=None, **kw):
    c = dict(kind=kind, R=32, hq=16, hk=0, budget=0, p_lo=512, p_hi=2048, page=64, q_scale=1.0, rows=0,
             dim=128, rot=128, at=0, layout="half", scaling="plain", new=False, salt=0)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a few interactive users, a tree each: launch latency
        _case("attn", "attn_tiny", R=4, hq=16, budget=16, p_lo=256, p_hi=256),
        # one GPU's 16 of a layer's 128 heads, single tokens, no drafts: bound by the cache's bytes
        _case("attn", "attn_decode_16h", R=64, hq=16, p_lo=1024, p_hi=8192, page=128),
        # the same share at high concurrency, trees of three slots on average
        _case("attn", "attn_tree_16h", R=128, hq=16, budget=256, p_lo=1024, p_hi=8192),
        # all 128 heads on each GPU (requests spread over the GPUs), an odd batch, sharper queries
        _case("attn", "attn_tree_128h", R=61, hq=128, budget=131, p_lo=1000, p_hi=4096, q_scale=2.0),
        # long documents: few requests, many verified nodes each
        _case("attn", "attn_long", R=16, hq=64, budget=192, p_lo=16384, p_hi=32768, page=256),
        # queries and keys of the verify slots of a 235B-class layer (64 / 4 heads)
        _case("rope", "rope_verify_235b", rows=384, hq=64, hk=4, p_hi=8192),
        # prompts of a batch of new chats, one layer of an 8B-class model, scaled for long contexts
        _case("rope", "rope_prompts_8b", rows=40000, hq=32, hk=8, p_hi=131072, scaling="smooth"),
        # the rotated part of latent attention's queries: 64 of a head's 192 dims, into the joined query
        _case("rope", "rope_latent_queries", rows=384, hq=128, dim=192, rot=64, at=128, layout="interleaved",
              scaling="bands", p_hi=160000),
        # prompts into the cache
        _case("store", "store_prompts", R=32, rows=40000, p_hi=4096, layout="interleaved", scaling="bands"),
        # the new rows of a verify step, beside the tree and nowhere else yet
        _case("store", "store_verify", R=128, rows=384, p_hi=8192, layout="interleaved", scaling="bands",
              new=True),
        # the accepted path of the large batch
        _case("commit", "commit_128", R=128, budget=256, p_lo=64, p_hi=512),
        # the same for a few users
        _case("commit", "commit_tiny", R=4, budget=16, p_lo=256, p_hi=300),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    kind = rng.choice(["attn", "attn", "attn", "rope", "rope", "store", "commit"])
    salt = rng.randrange(1 << 20)
    page = rng.choice([32, 64, 128, 256])
    layout = rng.choice(["half", "interleaved"])
    scaling = rng.choice(["plain", "linear", "smooth", "bands"])
    if kind == "attn":
        R = log_int(1, 128)
        hq = rng.choice([8, 16, 16, 20, 32, 40, 64, 128])
        budget = 0 if rng.random() < 0.35 else min(log_int(4, 256), 384 - R)
        p_hi = log_int(33, 32768)
        p_hi = max(1, int(min(p_hi, MAX_CACHE_BYTES / (R * ROW * 2.0),
                              MAX_FLOPS / (2.0 * (ROW + LATENT) * hq * (R + budget)))))
        return _case(kind, R=R, hq=hq, budget=budget, p_lo=rng.randint(max(1, p_hi // 8), p_hi), p_hi=p_hi,
                     page=page, q_scale=rng.choice([1.0, 1.0, 2.0]), salt=salt)
    if kind == "rope":
        hq, hk = rng.choice([(64, 4), (32, 8), (16, 1), (128, 0), (12, 3), (8, 8), (40, 5)])
        dim, rot, at = rng.choice([(128, 128, 0), (128, 64, 0), (192, 64, 128), (80, 80, 0), (96, 24, 0)])
        rows = max(1, min(log_int(1, 40000), int(MAX_ROPE_BYTES / (4.0 * (hq + hk) * rot))))
        return _case(kind, rows=rows, hq=hq, hk=hk, dim=dim, rot=rot, at=at, layout=layout, scaling=scaling,
                     p_hi=log_int(64, 1 << 20), salt=salt)
    if kind == "store":
        return _case(kind, R=log_int(1, 128), rows=log_int(1, MAX_STORE_ROWS), p_hi=log_int(64, 1 << 17), page=page,
                     layout=layout, scaling=scaling, new=rng.random() < 0.4, salt=salt)
    R = log_int(1, 256)
    p_hi = log_int(2, 1024)
    return _case(kind, R=R, budget=log_int(4, 256), p_lo=rng.randint(0, p_hi), p_hi=p_hi, page=page, salt=salt)


# ---- inputs ---------------------------------------------------------------

def _frequencies(rot, scaling):
    """Inverse frequencies (float64) and the factor on cosines and sines: base 10000, or
    500000 for the tables scaled to long contexts."""
    base = 10000.0 if scaling in ("plain", "linear", "bands") else 500000.0
    f = base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if scaling == "linear":  # positions pressed together
        return f / 4.0, 1.0
    if scaling == "smooth":  # long waves stretched by 8, short ones kept, a ramp between them
        turns = 8192.0 * f / (2 * math.pi)
        keep = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        return keep * f + (1 - keep) * f / 8.0, 1.0
    if scaling == "bands":  # stretched by 40: a ramp over the dims, and sharper scores
        def dim_of(n):
            return rot * math.log(4096.0 / (n * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(dim_of(32.0)), 0), min(math.ceil(dim_of(1.0)), rot - 1)
        ramp = np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        return f / 40.0 * ramp + f * (1 - ramp), 0.1 * math.log(40.0) + 1.0
    return f, 1.0


def _trees(R, budget, rng):
    """Slots of R drafted trees with `budget` nodes over all of them: offsets, masks and the
    parent slots (request-local)."""
    w = rng.gamma(2.0, 1.0, R)
    n = rng.multinomial(budget, w / w.sum())
    W = (int(n.max(initial=0)) + 1 + 31) // 32
    q_offsets = np.zeros(R + 1, np.int32)
    q_offsets[1:] = np.cumsum(n + 1)
    cap = R + budget
    mask, parent = np.zeros((cap, W), np.uint32), np.full(cap, -1, np.int32)
    for r in range(R):
        a = int(q_offsets[r])
        for j in range(int(n[r]) + 1):
            if j > 0:
                p = int(rng.integers(max(0, j - 4), j))
                parent[a + j] = p
                mask[a + j] = mask[a + p]
            mask[a + j, j >> 5] |= np.uint32(1 << (j & 31))
    return q_offsets, mask, parent


def _tables_of(tokens, page, rng, spare):
    """Block tables of shuffled pages for these capacities in tokens, and the pool's pages."""
    npg = (tokens.astype(np.int64) + page - 1) // page
    total = int(npg.sum()) + spare
    perm = rng.permutation(total).astype(np.int32)
    bt = np.full((len(tokens), max(1, int(npg.max()))), -1, np.int32)
    at = 0
    for r, k in enumerate(npg):
        bt[r, :k] = perm[at:at + k]
        at += int(k)
    return bt, total


def prepare(case, seed):
    rng = np.random.default_rng([seed, case["salt"], 29])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(rng.integers(1 << 62)))
    kind, R, hq, hk, page = case["kind"], case["R"], case["hq"], case["hk"], case["page"]
    # lengths belong to the case: another seed gives other values over the same sizes
    sizes = np.random.default_rng([case["salt"], R, case["p_hi"], case["rows"], 7])
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    s = dict(case, status=torch.zeros(1, dtype=torch.int32, device=DEV))

    def normal(*shape, scale=1.0):
        t = torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=gen)
        return t if scale == 1.0 else t.mul_(scale)

    if kind in ("rope", "store"):
        T = case["rows"]
        rot = ROPE if kind == "store" else case["rot"]
        f, factor = _frequencies(rot, case["scaling"])
        s.update(T=T, inv_freq=dev(f), factor=float(np.float32(factor)))
    if kind == "rope":
        dim, at = case["dim"], case["at"]
        s["positions"] = dev(rng.integers(0, case["p_hi"], T).astype(np.int32))
        s["x"] = {n: normal(T, h, dim) for n, h in (("q", hq), ("k", hk)) if h > 0}
        # where the rotated part goes: a place of its own, or the end of the joined query
        wide = ROW if at > 0 else rot
        s["y"] = {n: torch.zeros((T, h, wide), dtype=torch.bfloat16, device=DEV) for n, h in (("q", hq), ("k", hk))
                  if h > 0}
        s["wide"] = wide
        return s
    if kind == "store":
        # T rows of the batch's requests, one after another; the projection's output holds other columns too
        n = np.diff(np.concatenate([[0], np.sort(sizes.integers(0, T + 1, R - 1)), [T]])).astype(np.int64)
        P = sizes.integers(0, case["p_hi"] + 1, R)
        r = np.repeat(np.arange(R), n)
        pos = P[r] + np.arange(T) - np.repeat(np.cumsum(n) - n, n)
        s["positions"] = dev(pos.astype(np.int32))
        s["kv"] = normal(T, ROW + 64, scale=0.7)[:, :ROW]
        s["weight"] = (normal(LATENT) * 0.1 + 1.0).to(torch.bfloat16)
        if case["new"]:
            s["latent_new"] = torch.zeros((T, ROW), dtype=torch.bfloat16, device=DEV)
            return s
        local = P % page  # the pages before a request's first new row take no part
        bt, total = _tables_of(local + n, page, rng, 3)
        at = local[r] + pos - P[r]
        s["slot_map"] = dev(bt[r, at // page].astype(np.int64) * page + at % page)
        s["pages"] = normal(total, page, ROW)
        return s

    P = sizes.integers(case["p_lo"], case["p_hi"] + 1, R).astype(np.int32)
    q_offsets, mask, parent = _trees(R, case["budget"], sizes)
    cap = R + case["budget"]
    bt, total = _tables_of(P + (MAX_DEPTH + 1 if kind == "commit" else 0), page, rng, 3)
    s.update(cap=cap, W=mask.shape[1], most_slots=int(np.diff(q_offsets).max()), max_pages=bt.shape[1], total=total,
             block_table=dev(bt), prefix_len=dev(P), q_offsets=dev(q_offsets), tree_mask=dev(mask.view(np.int32)),
             pages=normal(total, page, ROW), latent_new=normal(cap, ROW))
    if kind == "attn":
        # scores of the scale that the expanded heads (192 dims) would have
        s.update(q=normal(cap, hq, ROW, scale=case["q_scale"] * math.sqrt(192.0 / ROW)), most_keys=int(P.max()),
                 sm_scale=float(np.float32(1.0 / math.sqrt(192.0))),
                 out=torch.zeros((cap, hq, LATENT), dtype=torch.bfloat16, device=DEV),
                 lse=torch.zeros((cap, hq), dtype=torch.float32, device=DEV))
        return s
    # commit: a path from the root to a random node of each tree
    acc_len, acc = np.zeros(R, np.int32), np.full((R, MAX_DEPTH), -1, np.int32)
    for r in range(R):
        a, b = int(q_offsets[r]), int(q_offsets[r + 1])
        j, path = int(sizes.integers(0, b - a)), []
        while j > 0:
            path.append(a + j)
            j = int(parent[a + j])
        path = path[::-1][:MAX_DEPTH]
        acc_len[r] = len(path)
        acc[r, :len(path)] = path
    s.update(accept_len=dev(acc_len), accept_slots=dev(acc), new_len=dev(np.zeros(R, np.int32)))
    return s


# ---- the operators' plain forms ---------------------------------------------

def _rotate(s, x, n):
    """x [rows, ..., n] rotated by its rows' positions; angles in 64 bits."""
    angle = s["positions"].double()[:, None] * s["inv_freq"]
    shape = (angle.shape[0],) + (1,) * (x.dim() - 2) + (n // 2,)
    c, sn = ((f(angle) * s["factor"]).float().view(shape) for f in (torch.cos, torch.sin))
    x = x.float()
    if s["layout"] == "half":
        a, b = x[..., :n // 2], x[..., n // 2:]
        return torch.cat([a * c - b * sn, b * c + a * sn], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)


def _rope_plain(s):
    at, rot = s["at"], s["rot"]
    for n, x in s["x"].items():
        s["y"][n][..., s["wide"] - rot:] = _rotate(s, x[..., at:at + rot], rot).to(torch.bfloat16)
    return s["y"]


def _store_plain(s):
    x = s["kv"][:, :LATENT].float()
    c = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["weight"].float()
    row = torch.cat([c, _rotate(s, s["kv"][:, LATENT:], ROPE)], 1).to(torch.bfloat16)
    if s["new"]:
        s["latent_new"].copy_(row)
        return s["latent_new"]
    s["pages"].view(-1, ROW)[s["slot_map"]] = row
    return s["pages"]


def _attn_plain(s):
    """softmax(sm_scale q c) c over each request's cached rows and the tree's own, all
    requests padded to the longest."""
    R, hq, page, S = s["R"], s["hq"], s["page"], s["most_slots"]
    npg = max(1, (s["most_keys"] + page - 1) // page)
    Pm = npg * page
    a = s["q_offsets"].long()
    j = torch.arange(S, device=DEV)
    at = (a[:-1, None] + j).clamp(max=s["cap"] - 1)  # [R, S]
    there = j < (a[1:] - a[:-1])[:, None]
    rows = torch.cat([s["pages"][s["block_table"][:, :npg].clamp(0).long()].view(R, Pm, ROW),
                      s["latent_new"][at]], 1).float()  # [R, Pm + S, ROW]
    q = s["q"][at].float().view(R, S * hq, ROW)
    z = torch.matmul(q, rows.transpose(-1, -2).contiguous())
    z *= s["sm_scale"]
    words = s["tree_mask"][at][..., (j >> 5).clamp(max=s["W"] - 1)]
    see_tree = ((words >> (j & 31)) & 1).bool() & there[:, None, :]  # [R, S, S]
    see_tree = see_tree[:, :, None, :].expand(R, S, hq, S).reshape(R, S * hq, S)
    keys = torch.arange(Pm, device=DEV) < s["prefix_len"][:, None]
    z[..., :Pm].masked_fill_(~keys[:, None, :], -math.inf)
    z[..., Pm:].masked_fill_(~see_tree, -math.inf)
    m = z.amax(-1, keepdim=True).clamp(min=-1e30)
    p = z.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, rows[..., :LATENT].contiguous())
    o /= l.clamp(min=1e-38)
    lse = (m + l.log()).squeeze(-1)
    # back to slots
    i = torch.arange(s["cap"], device=DEV)
    r = torch.searchsorted(a[1:].contiguous(), i, right=True).clamp(max=R - 1)
    k = (i - a[r]).clamp(max=S - 1)
    live = i < a[R]
    o = o.view(R, S, hq, LATENT)[r, k]
    lse = lse.view(R, S, hq)[r, k]
    return dict(out=torch.where(live[:, None, None], o, 0.0).to(torch.bfloat16),
                lse=torch.where(live[:, None], lse, 0.0))


def _commit_plain(s):
    page = s["page"]
    j = torch.arange(MAX_DEPTH + 1, device=DEV)
    src = torch.cat([s["q_offsets"][:-1, None], s["accept_slots"]], 1).long()
    live = j <= s["accept_len"][:, None]
    pos = s["prefix_len"][:, None] + j
    pg = s["block_table"].gather(1, (pos // page).clamp(max=s["max_pages"] - 1).long()).long()
    slot = pg * page + pos % page
    # (what is not accepted rewrites the root's row)
    slot = torch.where(live, slot, slot[:, :1])
    src = torch.where(live, src, src[:, :1])
    s["pages"].view(-1, ROW)[slot.view(-1)] = s["latent_new"][src.view(-1)]
    return dict(pages=s["pages"], new_len=s["prefix_len"] + 1 + s["accept_len"])


# ---- the calls ------------------------------------------------------------

def _run_own(s):
    import paper_2604_09603_amd as echo
    kind = s["kind"]
    layout = echo.ROPE_HALF if s["layout"] == "half" else echo.ROPE_INTERLEAVED
    if kind == "rope":
        at, rot = s["at"], s["rot"]
        x = {n: t[..., at:at + rot] for n, t in s["x"].items()}
        y = {n: t[..., s["wide"] - rot:] for n, t in s["y"].items()}
        echo.echo_rope(x["q"], y["q"], x.get("k"), y.get("k"), s["positions"], s["T"], s["hq"], s["hk"], rot, layout,
                       s["inv_freq"], s["factor"], status=s["status"])
        return s["y"]
    if kind == "store":
        echo.echo_store_latent(s["kv"], s["weight"], EPS, s["positions"], s["inv_freq"], s["factor"], layout, s["T"],
                               LATENT, ROPE, s.get("latent_new"), s.get("slot_map"), s.get("pages"), s["page"],
                               status=s["status"])
        return s["latent_new"] if s["new"] else s["pages"]
    if kind == "attn":
        ws = s.get("workspace")
        if ws is None:  # kept with the batch's other buffers
            n = echo.tree_verify_attn_latent_workspace_size(s["R"], s["cap"], s["hq"], s["max_pages"])
            raw = torch.empty(n + 256, dtype=torch.uint8, device=DEV)
            off = (-raw.data_ptr()) % 256
            ws = s["workspace"] = raw[off:off + n]
        echo.echo_tree_verify_attn_latent(
            s["q"], s["latent_new"], s["pages"], s["page"], s["block_table"], s["prefix_len"], s["q_offsets"],
            s["tree_mask"], s["W"], s["R"], s["cap"], s["hq"], LATENT, ROPE, s["sm_scale"], s["out"], s["lse"], ws,
            status=s["status"])
        return dict(out=s["out"], lse=s["lse"])
    echo.echo_commit_latent(
        s["q_offsets"], s["accept_len"], s["accept_slots"], MAX_DEPTH, s["latent_new"], s["R"], s["cap"], LATENT, ROPE,
        s["pages"], s["page"], s["block_table"], s["prefix_len"], s["new_len"], status=s["status"])
    return dict(pages=s["pages"], new_len=s["new_len"])


def run(s):
    if own:
        return _run_own(s)
    return {"rope": _rope_plain, "store": _store_plain, "attn": _attn_plain, "commit": _commit_plain}[s["kind"]](s)


# ---- what a pass cannot do without ------------------------------------------

def work(case):
    kind, R, B = case["kind"], case["R"], case["budget"]
    if kind == "rope":
        n = float(case["rows"]) * (case["hq"] + case["hk"]) * case["rot"]
        return {"bytes": 4.0 * n + 4.0 * case["rows"] + 4.0 * case["rot"], "flops": 3.0 * n}
    if kind == "store":
        return {"bytes": case["rows"] * (4.0 * ROW + (4 if case["new"] else 12)) + 2.0 * LATENT,
                "flops": case["rows"] * (4.0 * LATENT + 3.0 * ROPE)}
    if kind == "commit":
        n = min(4.0, 1 + 0.5 * B / R)
        return {"bytes": R * n * 4.0 * ROW + 16.0 * R, "flops": R * n * ROW}
    P, rows = 0.5 * (case["p_lo"] + case["p_hi"]), R + B
    return {"bytes": 2.0 * ROW * (R * P + rows) + rows * case["hq"] * (2.0 * (ROW + LATENT) + 4),
            "flops": 2.0 * (ROW + LATENT) * case["hq"] * rows * (P + 0.5 * rows / R)}


# ---- the definitions in 64 bits ---------------------------------------------

def _exact_turn(x, positions, f, factor, layout):
    """Complex numbers x_a + i x_b times factor e^(i position f)."""
    n = x.shape[-1]
    ia = torch.arange(0, n, 2, device=DEV) if layout == "interleaved" else torch.arange(n // 2, device=DEV)
    ib = ia + (1 if layout == "interleaved" else n // 2)
    turn = torch.polar(torch.full_like(f, factor).expand(len(positions), -1).contiguous(),
                       torch.outer(positions.double(), f))
    if x.dim() == 3:
        turn = turn[:, None, :]
    z = torch.complex(x[..., ia].double(), x[..., ib].double()) * turn
    y = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    y[..., ia], y[..., ib] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    kind, page = s["kind"], s["page"]
    if kind == "rope":
        at, rot, got = s["at"], s["rot"], {}
        for n, x in s["x"].items():
            y = s["y"][n].double()
            y[..., s["wide"] - rot:] = _exact_turn(x[..., at:at + rot], s["positions"], s["inv_freq"], s["factor"],
                                                   s["layout"])
            got[n] = y
        return got
    if kind == "store":
        x = s["kv"].double()
        row = torch.empty((s["T"], ROW), dtype=torch.float64, device=DEV)
        norm = torch.linalg.vector_norm(x[:, :LATENT], dim=1, keepdim=True) / math.sqrt(LATENT)
        row[:, :LATENT] = x[:, :LATENT] / torch.hypot(norm, torch.full_like(norm, math.sqrt(EPS))) * s["weight"].double()
        row[:, LATENT:] = _exact_turn(x[:, LATENT:], s["positions"], s["inv_freq"], s["factor"], s["layout"])
        if s["new"]:
            return row
        pages = s["pages"].double()
        for lo in range(0, s["T"], 4096):
            slot = s["slot_map"][lo:lo + 4096]
            pages[slot // page, slot % page] = row[lo:lo + 4096]
        return pages
    q0 = s["q_offsets"].cpu().tolist()
    P = s["prefix_len"].cpu().tolist()
    if kind == "commit":
        pages = s["pages"].double()
        bt = s["block_table"].cpu().tolist()
        n, slots = s["accept_len"].cpu().tolist(), s["accept_slots"].cpu().tolist()
        for r in range(s["R"]):
            for j, src in enumerate([q0[r]] + slots[r][:n[r]]):
                p = P[r] + j
                pages[bt[r][p // page], p % page] = s["latent_new"][src].double()
        return dict(pages=pages, new_len=None)
    hq = s["hq"]
    out = torch.zeros((s["cap"], hq, LATENT), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["cap"], hq), dtype=torch.float64, device=DEV)
    bt = s["block_table"].long()
    for r in range(s["R"]):
        a, b = q0[r], q0[r + 1]
        n = b - a
        C = torch.cat([s["pages"][bt[r, :(P[r] + page - 1) // page]].view(-1, ROW)[:P[r]],
                       s["latent_new"][a:b]]).double()
        bits = s["tree_mask"][a:b].cpu().numpy().view(np.uint32).astype(np.int64)
        j = np.arange(n)
        see = torch.from_numpy(((bits[:, j >> 5] >> (j & 31)) & 1).astype(bool)).to(DEV)
        see = torch.cat([torch.ones((n, P[r]), dtype=torch.bool, device=DEV), see], 1)
        for i in range(n):
            K = C[see[i]]
            z = (s["q"][a + i].double() @ K.T.contiguous()) * s["sm_scale"]
            lse[a + i] = torch.logsumexp(z, 1)
            out[a + i] = torch.softmax(z, 1) @ K[:, :LATENT]
    return dict(out=out, lse=lse)
