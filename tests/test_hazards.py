"""The kernels whose tile copies and products are inline assembly owe no wait states: their listings, built here,
are read (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

from paper_2604_09603_amd import build
from tests import gfx950_hazards as hazards


def _listing(*lines):
    return "kernel:\n" + "\n".join(lines) + "\n\ts_endpgm\n"


@pytest.mark.parametrize("owes,lines", [
    (1, ["v_readlane_b32 s4, v1, 3", "s_mov_b32 m0, s9", "s_nop 0", "global_load_lds_dwordx4 v2, s[4:5]"]),
    (0, ["v_readlane_b32 s4, v1, 3", "s_mov_b32 m0, s9", "s_nop 3", "global_load_lds_dwordx4 v2, s[4:5] offset:128"]),
    (0, ["v_readlane_b32 s4, v1, 3", "s_add_u32 s4, s4, s6", "s_nop 0", "global_load_dwordx4 v[4:7], v2, s[4:5]"]),
    (1, ["s_mov_b32 m0, s9", "global_load_lds_dwordx4 v2, s[4:5]"]),
    (1, ["v_cmp_gt_i32_e64 s[4:5], v1, v2", "s_nop 3", "buffer_load_dword v1, v2, s[4:7], 0 offen"]),
    (0, ["v_cmp_gt_i32_e64 s[4:5], v1, v2", "s_nop 4", "buffer_load_dword v1, v2, s[4:7], 0 offen"]),
    (1, ["v_mov_b32_e32 v5, v1", "s_nop 0", "v_mfma_f32_32x32x16_bf16 a[0:15], v[4:7], v[8:11], a[0:15]"]),
    (1, ["v_accvgpr_write_b32 a3, v1", "s_nop 0", "v_mfma_f32_32x32x16_bf16 a[0:15], v[4:7], v[8:11], a[0:15]"]),
    (0, ["v_mov_b32_e32 v5, v1", "s_nop 1", "v_mfma_f32_32x32x16_bf16 a[0:15], v[4:7], v[8:11], a[0:15]"]),
    # over a branch, and over a loop's back edge
    (1, ["s_cbranch_scc0 .LBB0_2", "v_readfirstlane_b32 s5, v1", ".LBB0_2:", "s_nop 3", "global_load_dword v1, v2, s[4:5]"]),
    (1, ["s_nop 7", ".LBB0_1:", "global_load_dword v1, v2, s[4:5]", "v_readfirstlane_b32 s5, v1", "s_cbranch_scc1 .LBB0_1"]),
    (0, ["v_readfirstlane_b32 s5, v1", "s_branch .LBB0_3", ".LBB0_2:", "global_load_dword v1, v2, s[4:5]", ".LBB0_3:",
         "s_nop 4", "s_cbranch_scc1 .LBB0_2"])])
def test_what_a_listing_owes(owes, lines):
    found, _ = hazards.scan(_listing(*lines))
    assert bool(found) == bool(owes), found


@pytest.mark.parametrize("name", ["attn.hip", "attn_latent.hip", "attn_q8.hip", "probe.hip"])
def test_inline_assembly_owes_nothing(name, tmp_path):
    if shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"):
        pytest.skip("hipcc not found")
    out = tmp_path / "listing.s"
    res = subprocess.run([build._hipcc(), *build.FLAGS, *build.FILE_FLAGS.get(name, []), "--cuda-device-only", "-S",
                          os.path.join(build.CSRC, name), "-o", str(out)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    found, copies = hazards.scan(out.read_text())
    assert copies > 0 and not found, found[:10]
