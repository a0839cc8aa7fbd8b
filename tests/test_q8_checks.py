"""Host-side refusals of the 8-bit cache's calls and of the block tables (no GPU needed)."""
import ctypes
import os

import pytest

import paper_2604_09603_amd as pkg

P = ctypes.c_void_p
INVALID, UNSUPPORTED, WORKSPACE = pkg.ERR_INVALID_ARG, pkg.ERR_UNSUPPORTED, pkg.ERR_WORKSPACE


@pytest.fixture(autouse=True)
def _lib():
    if not os.path.exists(pkg.LIB_PATH):
        pytest.skip("libecho.so not built")


CACHE = dict(kv_format=0, k_pages=P(256), v_pages=P(256), k_scale=P(256), v_scale=P(256),
             num_pages=8, page_size=64)
BAD_CACHE = [(dict(kv_format=2), INVALID), (dict(kv_format=-1), INVALID), (dict(k_pages=None), INVALID),
             (dict(v_pages=None), INVALID), (dict(k_scale=None), INVALID), (dict(v_scale=None), INVALID),
             (dict(k_pages=P(264)), INVALID), (dict(v_scale=P(258)), INVALID), (dict(num_pages=0), INVALID),
             (dict(num_pages=-1), INVALID), (dict(num_pages=1 << 62), UNSUPPORTED),
             (dict(num_pages=1 << 25), UNSUPPORTED), (dict(page_size=0), INVALID),
             (dict(page_size=16), UNSUPPORTED), (dict(page_size=96), UNSUPPORTED),
             (dict(page_size=-(1 << 31)), INVALID), (dict(head_dim=64), UNSUPPORTED),
             (dict(hkv=0), INVALID)]


def _attn(**kw):
    a = dict(q=P(256), k_new=P(256), v_new=P(256), **CACHE, block_table=P(256), max_pages=4,
             prefix_len=P(256), q_offsets=P(256), tree_mask=P(256), mask_words=1, R=2, max_rows=4, hq=8,
             hkv=4, head_dim=128, scale=0.1, out=P(256), lse=None, ws=P(256), ws_bytes=None, status=None,
             stream=None)
    a.update(kw)
    if a["ws_bytes"] is None:
        a["ws_bytes"] = pkg.tree_verify_attn_paged_q8_workspace_size(2, 4, 8, 4, 4)
    return pkg.load().echo_tree_verify_attn_paged_q8(*a.values())


@pytest.mark.parametrize("bad,code", BAD_CACHE + [
    (dict(R=0), INVALID), (dict(R=4096), UNSUPPORTED), (dict(max_rows=-1), INVALID), (dict(hq=6), INVALID),
    (dict(mask_words=0), INVALID), (dict(max_pages=0), INVALID), (dict(max_pages=1 << 26), UNSUPPORTED),
    (dict(R=4000, max_pages=1 << 20, ws_bytes=1 << 60), UNSUPPORTED),
    (dict(num_pages=(1 << 25) - 1, page_size=32, hkv=512, hq=512), UNSUPPORTED),
    (dict(max_rows=1 << 23), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(q=None), INVALID), (dict(k_new=None), INVALID),
    (dict(v_new=P(8)), INVALID), (dict(q=P(8)), INVALID), (dict(out=P(264)), INVALID),
    (dict(out=None), INVALID), (dict(block_table=None), INVALID), (dict(prefix_len=None), INVALID),
    (dict(q_offsets=None), INVALID), (dict(tree_mask=None), INVALID), (dict(ws=None), INVALID),
    (dict(ws=P(128)), WORKSPACE), (dict(ws_bytes=1024), WORKSPACE)])
def test_attention_refuses(bad, code):
    assert _attn(**bad) == code


def test_attention_without_rows_is_nothing():
    assert _attn(max_rows=0) == pkg.OK


def test_workspace_sizes():
    size = pkg.tree_verify_attn_paged_q8_workspace_size
    assert size(2, 4, 8, 4, 4) > 0
    assert size(4095, 4, 8, 4, 1000) > size(4095, 4, 8, 4, 1)
    assert size(0, 4, 8, 4, 4) == 0 and size(2, 4, 8, 4, 0) == 0
    assert size(2, 4, 8, 4, 4, head_dim=64) == 0


def _store(**kw):
    a = dict(k=P(256), v=P(256), k_stride=512, v_stride=512, slot_map=P(256), num_rows=3, hkv=4,
             head_dim=128, **CACHE, status=None, stream=None)
    a.update(kw)
    return pkg.load().echo_store_kv_q8(*a.values())


@pytest.mark.parametrize("bad,code", BAD_CACHE + [
    (dict(num_rows=-1), INVALID), (dict(k=None), INVALID), (dict(v=P(8)), INVALID),
    (dict(slot_map=None), INVALID), (dict(k_stride=504), INVALID), (dict(v_stride=516), INVALID),
    (dict(k_stride=1 << 31), UNSUPPORTED), (dict(v_stride=-512), INVALID)])
def test_store_refuses(bad, code):
    assert _store(**bad) == code


def test_store_without_rows_is_nothing():
    assert _store(num_rows=0, k=None, v=None, slot_map=None) == pkg.OK


def _commit(**kw):
    a = dict(q_offsets=P(256), accept_len=P(256), accept_slots=P(256), max_depth=4, k_new=P(256),
             v_new=P(256), R=2, max_rows=4, hkv=4, head_dim=128, **CACHE, block_table=P(256), max_pages=4,
             prefix_len=P(256), new_len=P(256), status=None, stream=None)
    a.update(kw)
    return pkg.load().echo_commit_kv_q8(*a.values())


@pytest.mark.parametrize("bad,code", BAD_CACHE + [
    (dict(R=0), INVALID), (dict(R=4096), UNSUPPORTED), (dict(max_rows=-1), INVALID),
    (dict(max_depth=0), UNSUPPORTED), (dict(max_depth=17), UNSUPPORTED), (dict(max_pages=0), INVALID),
    (dict(q_offsets=None), INVALID), (dict(accept_len=None), INVALID), (dict(accept_slots=None), INVALID),
    (dict(k_new=None), INVALID), (dict(v_new=P(258)), INVALID), (dict(block_table=None), INVALID),
    (dict(prefix_len=None), INVALID), (dict(new_len=None), INVALID)])
def test_commit_refuses(bad, code):
    assert _commit(**bad) == code


def _tables(**kw):
    a = dict(want_len=P(256), R=2, page_size=16, block_table=P(256), max_pages=4, num_held=P(256),
             num_held_out=P(256), free_pages=P(256), max_free=8, num_free=P(256), num_free_out=P(256),
             row_offsets=P(256), row_start=P(256), max_rows=4, slot_map=P(256), status=None, stream=None)
    a.update(kw)
    return pkg.load().echo_build_block_tables(*a.values())


@pytest.mark.parametrize("bad,code", [
    (dict(R=0), INVALID), (dict(R=4096), UNSUPPORTED), (dict(page_size=0), INVALID),
    (dict(page_size=24), UNSUPPORTED), (dict(max_pages=0), INVALID), (dict(max_pages=1 << 30), UNSUPPORTED),
    (dict(max_free=0), INVALID), (dict(want_len=None), INVALID), (dict(block_table=None), INVALID),
    (dict(num_held=None), INVALID), (dict(num_held_out=None), INVALID), (dict(free_pages=None), INVALID),
    (dict(num_free=None), INVALID), (dict(num_free_out=None), INVALID), (dict(max_rows=-1), INVALID),
    (dict(row_offsets=None), INVALID), (dict(row_start=None), INVALID)])
def test_tables_refuse(bad, code):
    assert _tables(**bad) == code


def test_status_bit_matches_the_header():
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                           "echo.h")) as f:
        text = f.read()
    from oracle import status as st
    assert "#define ECHO_DATA_NO_PAGES (1 << 8)" in text
    assert pkg.DATA_NO_PAGES == st.NO_PAGES == 1 << 8
    assert f"#define ECHO_KV_E4M3 {pkg.KV_E4M3}" in text and f"#define ECHO_KV_E5M2 {pkg.KV_E5M2}" in text
    assert f"#define ECHO_KV_BLOCK {pkg.KV_BLOCK}" in text
