"""Attention over values near the smallest normal number, where rows are merged from partial sums."""
import numpy as np
import pytest

from tests import gpu_common as gc

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    gc.require_gpu()


@pytest.mark.parametrize("R,hq,hkv,slots,keys", [(1, 8, 8, 1, 5000), (3, 16, 2, 4, 3000), (300, 64, 1, 3, 2016), (5, 128, 2, 4, 4000)])
@pytest.mark.parametrize("exponent", [-126, -124, -110])
def test_values_near_the_smallest_number(R, hq, hkv, slots, keys, exponent):
    """All logits are zero and all values of a dimension the same, +-2^exponent or 0: so is the output, whatever
    the kernel and the cut.  Sums are exact; a partial's rounding to fp16 is at most 2^-11 of it and the division
    2^-23, of numbers that may be subnormal (2^-149)."""
    import torch
    import paper_2604_09603_amd as pkg
    from paper_2604_09603_amd.step import _aligned_workspace
    nq = R * slots
    v = torch.full((128,), 2.0 ** exponent, device="cuda:0")
    v[::3] *= -1
    v[::4] = 0
    bits = lambda t: t.contiguous().view(torch.int16)  # noqa: E731
    zeros = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda:0")  # noqa: E731
    mask = torch.from_numpy(np.tile((2 << np.arange(slots)) - 1, R).astype(np.int32)).to("cuda:0")
    kvo = torch.arange(R + 1, dtype=torch.int64, device="cuda:0") * keys
    qo = torch.arange(R + 1, dtype=torch.int32, device="cuda:0") * slots
    out = torch.full((nq, hq, 128), 7.0, device="cuda:0")
    ws = _aligned_workspace(pkg.tree_verify_attn_workspace_size(R, nq, hq, hkv), "cuda:0")
    print(f"[small values] R={R} heads {hq}/{hkv} slots {slots} keys {keys} 2^{exponent}", flush=True)
    pkg.echo_tree_verify_attn(bits(zeros(nq, hq, 128)), bits(zeros(nq, hkv, 128)),
                              bits(v.bfloat16().expand(nq, hkv, 128)), bits(zeros(R * keys, hkv, 128)),
                              bits(v.bfloat16().expand(R * keys, hkv, 128)), kvo, R * keys, qo, mask, 1, R, nq, hq, hkv,
                              128, 1.0, out, None, ws)
    torch.cuda.synchronize()
    err = (out.double() - v.double()).abs()
    assert bool((err <= v.double().abs() * (2.0 ** -11 + 2.0 ** -22) + 2.0 ** -148).all()), float(err.max() / 2.0 ** exponent)
