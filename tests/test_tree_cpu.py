"""Refusals and sizes of the paged calls on a machine without a GPU: planner handles run every check of the arguments."""
import os
import shutil
import subprocess

import pytest

import paper_2506_18879_amd as cv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, CONFIG, SHAPE, WORKSPACE, NO_DEVICE = 1, 2, 3, 4, 6
P = 1 << 20     # an address that is aligned and never read


def cfg(**kw):
    c = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, m_key=16, m_val=32, k=256, q_dtype=1, codebook_dtype=1, rope_base=500000.0, softmax_scale=0.0,
             max_position=131072)
    c.update(kw)
    return cv.Config(**c)


@pytest.fixture
def planner():
    made = []

    def make(**kw):
        made.append(cv.commvq_create_planner(cfg(**kw)))
        return made[-1]
    yield make
    for h in made:
        cv.commvq_destroy(h)


def status(call, *args):
    with pytest.raises(cv.CommVQError) as e:
        call(*args)
    return e.value.status


def attn(h, pages=None, tables=P, ws=P, ws_bytes=None, swap=None, **kw):
    t = dict(batch=2, total_nodes=20, max_nodes=12, max_seqlen=5000, seq_lens=P, block_tables=P, cu_nodes=P, node_pos=P, node_mask=P, key_pos=None,
             pair_axis=None)
    t.update(kw)
    pages = pages or cv.make_pages(16, 1000, 400)
    if ws_bytes is None:
        ws_bytes = 1 << 40
    args = dict(q=P, node_keys=P, node_vals=P, key_pages=P, val_pages=P, key_codebooks=P, val_codebooks=P, tables=tables, out=P)
    args.update(swap or {})
    return status(cv.commvq_tree_attn, h, pages, cv.make_tree(**t), *args.values(), ws, ws_bytes, 0)


def test_what_is_acceptable_stops_only_at_the_missing_device(planner):
    h = planner()
    assert attn(h) == NO_DEVICE
    assert attn(h, tables=None) == NO_DEVICE
    assert attn(h, node_mask=None) == NO_DEVICE
    assert attn(h, max_seqlen=0) == NO_DEVICE
    assert attn(h, total_tokens=5000) == NO_DEVICE and attn(h, total_tokens=10000) == NO_DEVICE
    assert attn(h, q_stride=48 * 128, node_stride=48 * 128) == NO_DEVICE
    assert attn(h, pages=cv.make_pages(1024, 1000, 400, 3), pair_axis=[0] * 16 + [1] * 24 + [2] * 24, key_pos=P) == NO_DEVICE
    assert attn(planner(q_dtype=0, codebook_dtype=0), tables=None) == NO_DEVICE
    assert attn(planner(position_free=1)) == NO_DEVICE
    assert status(cv.commvq_tree_prepare, h, P, P, P) == NO_DEVICE
    assert status(cv.commvq_store_pages, h, cv.make_pages(16, 10, 1), 5, P, P, P, P, P, P, P) == NO_DEVICE
    assert status(cv.commvq_store_pages, h, cv.make_pages(16, 10, 1), 5, P, P, P, None, P, P, None) == NO_DEVICE


@pytest.mark.parametrize("kw", [dict(seq_lens=None), dict(block_tables=None), dict(cu_nodes=None), dict(node_pos=None), dict(ws=None)])
def test_missing_pointers(planner, kw):
    assert attn(planner(), **kw) == (WORKSPACE if "ws" in kw else NULL)


def test_missing_data(planner):
    h = planner()
    for name in ("q", "node_keys", "node_vals", "key_pages", "val_pages", "key_codebooks", "val_codebooks", "out"):
        assert attn(h, swap={name: None}) == NULL
        assert attn(h, swap={name: P + 8}) == SHAPE
    assert attn(h, tables=P + 8) == SHAPE
    assert attn(h, pages=cv.make_pages(16, 1000, 400, 2)) == NULL         # two axes and no map


@pytest.mark.parametrize("pages", [(8, 10, 10), (24, 10, 10), (2048, 10, 10), (0, 10, 10), (16, 0, 10), (16, 1 << 27, 400), (16, 10, 0), (16, 1000, 400, 0), (16, 1000, 400, 5)])
def test_pool_geometry(planner, pages):
    h, pages = planner(), cv.make_pages(*pages)
    assert attn(h, pages=pages) == SHAPE
    assert status(cv.commvq_store_pages, h, pages, 1, P, P, P, None, P, P, None) == SHAPE
    assert status(cv.commvq_page_tables, pages, 1, P, P, P, 1, P, P, P, P, P, 1, P) == SHAPE


@pytest.mark.parametrize("kw", [dict(batch=0), dict(max_nodes=0), dict(max_nodes=65, total_nodes=70), dict(total_nodes=11), dict(total_nodes=25), dict(max_seqlen=-1),
                                dict(max_seqlen=6401), dict(q_stride=4095), dict(q_stride=4100), dict(q_stride=8), dict(node_stride=1020), dict(node_stride=1028),
                                dict(q_stride=-4096), dict(total_tokens=-1), dict(total_tokens=4999), dict(total_tokens=10001)])
def test_shapes(planner, kw):
    assert attn(planner(), **kw) == SHAPE


def test_positions_and_axes(planner):
    assert attn(planner(max_position=4000)) == SHAPE                      # implicit positions beyond the phase tables
    assert attn(planner(max_position=4000), key_pos=P) == NO_DEVICE
    assert attn(planner(max_position=4000, position_free=1)) == NO_DEVICE
    assert attn(planner(), pages=cv.make_pages(16, 1000, 400, 2), pair_axis=[0] * 63 + [2]) == SHAPE
    with pytest.raises(ValueError):
        cv.make_tree(1, 1, 1, 1, P, P, P, P, pair_axis=[0] * 63)


def test_formats(planner):
    paired = planner(key_format=cv.COMMVQ_KEYS_PAIRED, key_levels=11)
    binary = planner(value_format=cv.COMMVQ_VALUES_BINARY, value_bits=1024)
    for h in (paired, binary):
        assert attn(h) == CONFIG
        assert status(cv.commvq_tree_workspace_bytes, h, 1, 1, 1, 10) == CONFIG
        assert status(cv.commvq_tree_table_bytes, h) == CONFIG
        assert status(cv.commvq_tree_prepare, h, P, P, P) == CONFIG
        assert status(cv.commvq_store_pages, h, cv.make_pages(16, 10, 1), 5, P, P, P, None, P, P, None) == CONFIG
    f32 = planner(q_dtype=0, codebook_dtype=0)
    assert attn(f32) == CONFIG and status(cv.commvq_tree_table_bytes, f32) == CONFIG   # tables are for bf16 codebooks


def test_workspace(planner):
    h = planner()
    need = cv.commvq_tree_workspace_bytes(h, 2, 20, 12, 5000)
    assert need % 256 == 0 and attn(h, ws_bytes=need) == NO_DEVICE
    assert attn(h, ws_bytes=need - 1) == WORKSPACE and attn(h, ws=P + 128) == WORKSPACE
    assert cv.commvq_tree_workspace_bytes(h, 1, 1, 1, 0) > 0
    for bad in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 2, 1, 1), (1, 65, 65, 1), (1, 1, 1, -1)):
        assert status(cv.commvq_tree_workspace_bytes, h, *bad) == SHAPE
    assert cv.commvq_tree_table_bytes(h) == 8 * (16 + 32) * 256 * 128 * 2 + 256   # and a power of two per head and kind
    assert status(cv.commvq_tree_prepare, h, P, P, P + 8) == SHAPE and status(cv.commvq_tree_prepare, h, None, P, P) == NULL


def test_stores_and_tables(planner):
    h, pages = planner(), cv.make_pages(16, 10, 4)
    ok = [5, P, P, P, P, P, P, P]
    for i in (1, 2, 3, 5, 6):
        assert status(cv.commvq_store_pages, h, pages, *(ok[:i] + [None] + ok[i + 1:])) == NULL
    for i in (4, 7):                                                      # positions come with the pool's positions
        assert status(cv.commvq_store_pages, h, pages, *(ok[:i] + [None] + ok[i + 1:])) == NULL
    for i in (2, 3, 5, 6):
        assert status(cv.commvq_store_pages, h, pages, *(ok[:i] + [P + 4] + ok[i + 1:])) == SHAPE
    assert status(cv.commvq_store_pages, h, pages, 0, *ok[1:]) == SHAPE
    assert status(cv.commvq_store_pages, h, pages, 1 << 30, *ok[1:]) == SHAPE
    good = [2, P, P, P, 3, P, P, P, P, P, 7, P]
    for i in (1, 2, 3, 5, 6, 7, 8, 11):
        assert status(cv.commvq_page_tables, pages, *(good[:i] + [None] + good[i + 1:])) == NULL
    for i, v in ((0, 0), (4, -1), (10, -1), (10, (1 << 30) + 1)):
        assert status(cv.commvq_page_tables, pages, *(good[:i] + [v] + good[i + 1:])) == SHAPE


def test_host_code_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    hipcc, clang = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "/opt/rocm/lib/llvm/bin/clang"
    driver = os.path.join(ROOT, "tests", "sanitize", "pages_driver.c")
    if not (os.path.exists(hipcc) and os.path.exists(clang) and shutil.which(clang)) or not os.path.exists(driver):
        pytest.skip("no hipcc")
    src = [os.path.join(ROOT, "paper_2506_18879_amd", "csrc", "commvq%s.hip" % f) for f in ("", "_encode", "_em", "_vbits", "_pages", "_tree")]
    run = lambda cmd: subprocess.run(cmd, check=True, capture_output=True, text=True).stdout
    run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-shared", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
         "-I" + os.path.join(ROOT, "include"), "-o", str(tmp_path / "libcommvq_san.so"), *src])
    exe = str(tmp_path / "pages_driver")
    run([clang, "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I" + os.path.join(ROOT, "include"), "-o", exe, driver,
         "-L" + str(tmp_path), "-lcommvq_san", "-Wl,-rpath," + str(tmp_path)])
    assert "pages_driver: ok" in run([exe])
