"""The 8-bit paged cache where its calls can go wrong: their limits."""
import pytest

from oracle import kvq8, status as st
from tests import gpu_common as gc
from tests.test_gpu_kvq8 import _log, _zeros

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
