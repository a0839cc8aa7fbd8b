"""The latent operators together, as an engine uses them: pages from a pool, prompts into the cache, then
steps of a drafted tree per request (queries rotated, new rows beside the tree, attention,
acceptance, commit), eagerly against the oracle and as a captured step that is replayed."""
import numpy as np
import pytest

from oracle import latent
from tests import gpu_common as gc
from tests.test_gpu_latent import _bf, _bits, _dev, _log, _rotated_ok, _rows_ok, _zeros
from tests.test_gpu_latent_attn import _check

pytestmark = pytest.mark.gpu
HQ, PS, DEPTH, NOPE = 16, 32, 4, 128
SCALE = 192 ** -0.5
PROMPTS = [40, 1, 31, 100, 64]
# each request's tree: parents (request-local), a token per node
TREES = [[-1, 0, 0, 1, 3], [-1], [-1, 0, 1, 2, 3, 0], [-1, 0], [-1, 0, 0, 0, 2, 2]]
EPS = 1e-6


@pytest.fixture(autouse=True)
def _need_gpu():
    gc.require_gpu()


class Engine:
    """The buffers of a batch, and a step over them."""

    def __init__(self):
        import torch
        import paper_2604_09603_amd as pkg
        from paper_2604_09603_amd.step import _aligned_workspace
        rng = np.random.default_rng(77)
        self.R, n = len(PROMPTS), [len(t) for t in TREES]
        self.qo = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.cap = int(self.qo[-1]) + 2
        self.mask = np.zeros((self.cap, 1), np.uint32)
        parent, depth = np.full(self.cap, -1, np.int32), np.zeros(self.cap, np.int32)
        req = np.zeros(self.cap, np.int32)
        for r, t in enumerate(TREES):
            for j, p in enumerate(t):
                s = self.qo[r] + j
                req[s] = r
                if p >= 0:
                    parent[s], depth[s] = p, depth[self.qo[r] + p] + 1
                    self.mask[s] = self.mask[self.qo[r] + p]
                self.mask[s, 0] |= np.uint32(1 << j)
        self.parent = parent
        self.f, self.factor = pkg.echo_rope_frequencies(64, 10000.0, "bands", 40.0, 4096.0)
        self.weight = _bf(1 + 0.1 * rng.standard_normal(512))
        self.pages = torch.full((64, PS, 576), float("nan"), dtype=torch.bfloat16, device="cuda:0")
        self.bt = torch.full((self.R, 8), -1, dtype=torch.int32, device="cuda:0")
        self.held, self.free, self.nfree = _zeros(self.R), _dev(rng.permutation(64).astype(np.int32)), _zeros(1) + 64
        self.plen, self.status = _zeros(self.R), _zeros(1)
        self.dqo, self.dmask, self.dparent = _dev(self.qo), _dev(self.mask), _dev(parent)
        self.ddepth, self.dreq, self.df, self.dweight = _dev(depth), _dev(req), _dev(np.array(self.f)), _dev(self.weight)
        self.positions, self.want = _zeros(self.cap), _zeros(self.R)
        self.qkv = torch.zeros((self.cap, HQ, NOPE + 64), dtype=torch.bfloat16, device="cuda:0")
        self.q = torch.zeros((self.cap, HQ, 576), dtype=torch.bfloat16, device="cuda:0")
        self.kv = torch.zeros((self.cap, 640), dtype=torch.bfloat16, device="cuda:0")
        self.new = torch.full((self.cap, 576), float("nan"), dtype=torch.bfloat16, device="cuda:0")
        self.out = torch.full((self.cap, HQ, 512), float("nan"), dtype=torch.bfloat16, device="cuda:0")
        self.lse = torch.full((self.cap, HQ), float("nan"), dtype=torch.float32, device="cuda:0")
        self.token, self.target = _zeros(self.cap), _zeros(self.cap)
        self.alen, self.aslots, self.bonus = _zeros(self.R), _zeros(self.R, DEPTH), _zeros(self.R)
        self.ws = _aligned_workspace(pkg.tree_verify_attn_latent_workspace_size(self.R, self.cap, HQ, 8), "cuda:0")
        self.rng = rng

    def pages_for(self, want, **kw):
        import paper_2604_09603_amd as pkg
        pkg.echo_build_block_tables(want, self.R, PS, self.bt, self.held, self.held, self.free, self.nfree, self.nfree,
                                    status=self.status, **kw)

    def prompts(self):
        import torch
        import paper_2604_09603_amd as pkg
        T = sum(PROMPTS)
        at = np.concatenate([[0], np.cumsum(PROMPTS)]).astype(np.int32)
        kv = _bf(self.rng.standard_normal((T, 576)))
        pos = np.concatenate([np.arange(n) for n in PROMPTS]).astype(np.int32)
        slots = torch.zeros(T, dtype=torch.int64, device="cuda:0")
        self.pages_for(_dev(np.array(PROMPTS, np.int32)), row_offsets=_dev(at), row_start=_zeros(self.R), slot_map=slots)
        pkg.echo_store_latent(_dev(kv), self.dweight, EPS, _dev(pos), self.df, self.factor, pkg.ROPE_INTERLEAVED, T, 512,
                              64, None, slots, self.pages, PS, status=self.status)
        self.plen.copy_(_dev(np.array(PROMPTS, np.int32)))
        got = _bits(self.pages.view(-1, 576)[slots])
        _rows_ok(got, kv, self.weight, EPS, pos, np.array(self.f), self.factor, 1)

    def inputs(self, k):
        """A step's inputs: they depend on nothing but k."""
        rng = np.random.default_rng(1000 + k)
        self.qkv.copy_(_dev(_bf(rng.standard_normal(self.qkv.shape))))
        self.q[..., :512].copy_(_dev(_bf(rng.standard_normal((self.cap, HQ, 512)) * 0.3)))
        self.kv.copy_(_dev(_bf(rng.standard_normal(self.kv.shape))))
        self.token.copy_(_dev(rng.integers(0, 3, self.cap).astype(np.int32)))
        self.target.copy_(_dev(rng.integers(0, 3, self.cap).astype(np.int32)))

    def step(self):
        import torch
        import paper_2604_09603_amd as pkg
        torch.add(self.plen, DEPTH + 1, out=self.want)
        self.pages_for(self.want)
        torch.add(self.plen[self.dreq.long()], self.ddepth, out=self.positions)
        rot = self.qkv[..., NOPE:], self.q[..., 512:]
        pkg.echo_rope(*rot, None, None, self.positions, self.cap, HQ, 0, 64, pkg.ROPE_INTERLEAVED, self.df, self.factor,
                      status=self.status)
        pkg.echo_store_latent(self.kv[:, :576], self.dweight, EPS, self.positions, self.df, self.factor,
                              pkg.ROPE_INTERLEAVED, self.cap, 512, 64, self.new, None, None, 0, status=self.status)
        pkg.echo_tree_verify_attn_latent(self.q, self.new, self.pages, PS, self.bt, self.plen, self.dqo, self.dmask, 1,
                                         self.R, self.cap, HQ, 512, 64, SCALE, self.out, self.lse, self.ws,
                                         status=self.status)
        pkg.echo_accept(self.dqo, self.dparent, self.token, self.target, self.R, self.cap, DEPTH, self.alen, self.aslots,
                        self.bonus, status=self.status)
        pkg.echo_commit_latent(self.dqo, self.alen, self.aslots, DEPTH, self.new, self.R, self.cap, 512, 64, self.pages,
                               PS, self.bt, self.plen, self.plen, status=self.status)

    def state(self):
        import torch
        torch.cuda.synchronize()
        return [_bits(t) for t in (self.pages, self.new, self.q, self.out)] + [
            t.cpu().numpy() for t in (self.plen, self.bt, self.lse, self.alen, self.aslots, self.bonus, self.status)]


def test_steps_match_the_oracle():
    e = Engine()
    e.prompts()
    accepted = 0
    for k in range(6):
        _log(f"[latent run] step {k}")
        e.inputs(k)
        plen, pages = e.plen.cpu().numpy(), _bits(e.pages)
        e.step()
        live = int(e.qo[-1])
        pos = e.positions.cpu().numpy()[:live]
        f, new = np.array(e.f), _bits(e.new)
        _rows_ok(new[:live], _bits(e.kv)[:live, :576], e.weight, EPS, pos, f, e.factor, 1)
        _rotated_ok(_bits(e.q)[:live, :, 512:], latent.bf16_to_f64(_bits(e.qkv)[:live, :, NOPE:]), pos, f, e.factor, 1)
        bt = e.bt.cpu().numpy()
        assert int(e.status.item()) == 0
        _check(dict(q=_bits(e.q), new=new, pages=pages, bt=bt, plen=plen, qo=e.qo, mask=e.mask, hq=HQ, scale=SCALE,
                    cap=e.cap), e.out.float().cpu().numpy(), e.lse.cpu().numpy(), 0)
        alen, aslots = e.alen.cpu().numpy(), e.aslots.cpu().numpy()
        token, target = e.token.cpu().numpy(), e.target.cpu().numpy()
        for r in range(e.R):  # the path that was accepted is one of the tree's, and matches
            at = e.qo[r]
            for s in aslots[r, :alen[r]]:
                assert e.qo[r] + e.parent[s] == at and token[s] == target[at]
                at = s
        want, wl, _ = latent.commit_latent(e.qo, alen, aslots, new, pages, bt, plen)
        assert np.array_equal(_bits(e.pages), want) and np.array_equal(e.plen.cpu().numpy(), wl)
        accepted += int(alen.sum())
    assert accepted > 0


def test_captured_steps_match_eager_ones():
    import torch
    eager, captured = Engine(), Engine()
    want = []
    eager.prompts()
    for k in range(4):
        eager.inputs(k)
        eager.step()
        want.append(eager.state())
    captured.inputs(0)  # (a warm-up over an empty cache, with lengths put back)
    captured.step()
    torch.cuda.synchronize()
    fresh = Engine()
    for name in ("pages", "bt", "held", "free", "nfree", "plen", "status", "new", "out", "lse"):
        getattr(captured, name).copy_(getattr(fresh, name))
    captured.rng = fresh.rng
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    captured.prompts()
    for k in range(4):
        captured.inputs(k)
        x = torch.randn(512, 512, device="cuda:0")
        (x @ x).sum().item()
        graph.replay()
        for a, b in zip(captured.state(), want[k]):
            assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f")
