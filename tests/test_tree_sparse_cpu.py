"""Draft trees and sparse decoding without a GPU: refusals (every bad argument is answered before any CUDA call) and the shares of the
tree kernel's CTAs."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2607_09207_b200 import build as pd_build
from paper_2607_09207_b200 import pdattn


@pytest.fixture(scope="module", autouse=True)
def _built():
    pd_build.build()


P = 0x10000      # an aligned address that no call may touch


def step(**kw):
    a = pdattn.Args()
    for f in ("q", "k_cache", "v_cache", "out", "block_table", "context_lens", "workspace"):
        setattr(a, f, P)
    a.num_seqs, a.num_q_heads, a.num_kv_heads, a.head_dim, a.block_size = 3, 4, 2, 64, 16
    a.max_blocks_per_seq, a.num_blocks, a.scale = 4, 12, 0.1
    a.kv_block_stride, a.kv_head_stride, a.kv_token_stride = 2048, 1024, 64
    a.workspace_bytes = 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_STEPS = [(dict(num_seqs=-1), pdattn.INVALID_ARG), (dict(num_q_heads=5), pdattn.INVALID_ARG), (dict(head_dim=96), pdattn.UNSUPPORTED),
             (dict(block_size=8), pdattn.UNSUPPORTED), (dict(num_q_heads=34), pdattn.UNSUPPORTED), (dict(max_blocks_per_seq=0), pdattn.INVALID_ARG),
             (dict(num_blocks=0), pdattn.INVALID_ARG), (dict(workspace=P + 128), pdattn.MISALIGNED),
             (dict(workspace_bytes=8447), pdattn.WORKSPACE_TOO_SMALL)]
BAD_STEPS += [({f: None}, pdattn.INVALID_ARG) for f in ("q", "k_cache", "v_cache", "out", "block_table", "context_lens", "workspace")]
BAD_STEPS += [({f: P + 8}, pdattn.MISALIGNED) for f in ("q", "k_cache", "v_cache", "out")]
BAD_STRIDES = [(dict(kv_head_stride=0), pdattn.INVALID_ARG), (dict(kv_token_stride=56), pdattn.INVALID_ARG),
               (dict(kv_block_stride=2052), pdattn.UNSUPPORTED)]


def test_tree_refusals():
    L = pdattn.lib()
    n = pdattn.tree_workspace_size(4, 2, 64, 16, 64)
    assert n % 256 == 0 and n < pdattn.tree_workspace_size(4, 2, 128, 16, 64)
    for bad in ((5, 2, 64, 16, 8), (4, 2, 96, 16, 8), (4, 2, 64, 16, 65), (4, 2, 64, 16, 0)):
        with pytest.raises(pdattn.PdattnError):
            pdattn.tree_workspace_size(*bad)

    def both(cu=P, num=9, mask=P, top=8, ks=P, vs=P, **kw):
        a = step(**kw)
        return (L.pdattn_decode_tree(ctypes.byref(a), cu, num, mask, top, None),
                L.pdattn_decode_tree_fp8(ctypes.byref(a), cu, num, mask, top, ks, vs, None))
    assert L.pdattn_decode_tree(None, P, 9, P, 8, None) == L.pdattn_decode_tree_fp8(None, P, 9, P, 8, P, P, None) == pdattn.INVALID_ARG
    assert both(num=0) == both(num_seqs=0) == (pdattn.OK,) * 2                   # nothing to do
    for kw in (dict(num=-1), dict(cu=None), dict(mask=None), dict(top=0)):
        assert both(**kw) == (pdattn.INVALID_ARG,) * 2, kw
    assert both(top=65) == both(num_seqs=65537) == (pdattn.UNSUPPORTED,) * 2
    assert both(mask=P + 4) == (pdattn.MISALIGNED,) * 2
    assert both(workspace_bytes=n - 1) == (pdattn.WORKSPACE_TOO_SMALL,) * 2
    assert both(ks=None)[1] == both(vs=None)[1] == pdattn.INVALID_ARG
    for kw, why in BAD_STEPS:
        assert both(**kw) == (why,) * 2, kw
    for kw, why in BAD_STRIDES:
        assert both(**kw)[0] == why, kw


def test_accept_and_trim_refusals():
    L = pdattn.lib()

    def call(k=P, v=P, table=P, lens=P, cu=P, acc=P, cnt=P, m=8, S=3, H=2, d=64, bs=16, MB=4, NB=12, eb=2, sb=2048, sh=1024, st=64, ws=None):
        return L.pdattn_tree_accept(k, v, table, lens, cu, acc, cnt, m, S, H, d, bs, MB, NB, eb, sb, sh, st, ws, None)
    assert call(S=0) == call(m=0) == pdattn.OK
    for kw in (dict(k=None), dict(v=None), dict(table=None), dict(lens=None), dict(cu=None), dict(acc=None), dict(cnt=None), dict(m=-1),
               dict(S=-1), dict(H=0), dict(MB=0), dict(NB=0), dict(sb=0), dict(sh=-8), dict(st=56)):
        assert call(**kw) == pdattn.INVALID_ARG, kw
    for kw in (dict(m=65), dict(d=96), dict(bs=8), dict(eb=4), dict(sh=1028), dict(H=65536)):
        assert call(**kw) == pdattn.UNSUPPORTED, kw
    assert call(k=P + 8) == call(v=P + 4) == call(ws=P + 2) == pdattn.MISALIGNED
    n = pdattn.pages_workspace_size(12, 3)
    good = pdattn.PoolArgs(P, P, P, 12)

    def trim(pool=good, table=P, lens=P, new=P, S=3, MB=4, bs=16, ws=P, nb=n):
        return L.pdattn_pages_trim(ctypes.byref(pool) if pool is not None else None, table, lens, new, S, MB, bs, ws, nb, None)
    assert trim(S=0) == pdattn.OK
    for kw in (dict(pool=None), dict(pool=pdattn.PoolArgs(None, P, P, 12)), dict(table=None), dict(lens=None), dict(new=None), dict(S=-1),
               dict(MB=0), dict(bs=0), dict(ws=None)):
        assert trim(**kw) == pdattn.INVALID_ARG, kw
    assert trim(bs=24) == pdattn.UNSUPPORTED and trim(ws=P + 64) == pdattn.MISALIGNED and trim(nb=n - 1) == pdattn.WORKSPACE_TOO_SMALL


def test_rotation_positions_refusals():
    L = pdattn.lib()
    a = pdattn.RopeArgs()
    a.num_tokens, a.num_seqs, a.num_q_heads, a.num_kv_heads, a.head_dim, a.block_size, a.rotary_dim = 0, 0, 4, 2, 64, 16, 64
    assert L.pdattn_rope_append_at(ctypes.byref(a), P, None) == L.pdattn_rope_append_at_fp8(ctypes.byref(a), P, P, P, None) == pdattn.OK
    assert L.pdattn_rope_append_at(ctypes.byref(a), None, None) == pdattn.INVALID_ARG
    assert L.pdattn_rope_append_at_fp8(ctypes.byref(a), None, P, P, None) == pdattn.INVALID_ARG
    assert L.pdattn_rope_append_at(None, P, None) == pdattn.INVALID_ARG


def test_summary_refusals():
    L = pdattn.lib()

    def args(**kw):
        a = pdattn.SummaryArgs(P, P, P, P, 2, 64, 16, 12, 2, 2048, 1024, 64, None)
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    def both(table=P, lens=P, cu=P, num=9, S=3, MB=4, pages=P, count=5, **kw):
        a = args(**kw)
        return (L.pdattn_summarize_append(ctypes.byref(a), table, lens, cu, num, S, MB, None),
                L.pdattn_summarize_pages(ctypes.byref(a), pages, count, None))
    assert L.pdattn_summarize_append(None, P, P, P, 9, 3, 4, None) == L.pdattn_summarize_pages(None, P, 5, None) == pdattn.INVALID_ARG
    assert both(num=0, count=0) == (pdattn.OK,) * 2 and both(S=0)[0] == pdattn.OK
    for kw in (dict(k_cache=None), dict(codes=None), dict(exponents=None), dict(num_kv_heads=0), dict(num_blocks=0), dict(kv_block_stride=0),
               dict(kv_token_stride=56), dict(element_bytes=1, k_scale=None)):
        assert both(**kw) == (pdattn.INVALID_ARG,) * 2, kw
    for kw in (dict(head_dim=32), dict(block_size=48), dict(element_bytes=4), dict(kv_head_stride=1028)):
        assert both(**kw) == (pdattn.UNSUPPORTED,) * 2, kw
    for kw in (dict(k_cache=P + 8), dict(codes=P + 8), dict(workspace=P + 2)):
        assert both(**kw) == (pdattn.MISALIGNED,) * 2, kw
    for kw in (dict(table=None), dict(lens=None), dict(num=-1), dict(S=-1), dict(MB=0), dict(cu=None)):
        assert both(**kw)[0] == pdattn.INVALID_ARG, kw
    assert both(pages=None)[1] == both(count=-1)[1] == pdattn.INVALID_ARG


def test_select_refusals():
    L = pdattn.lib()
    n = pdattn.select_workspace_size(3, 2, 40)
    for bad in ((-1, 2, 40), (3, 0, 40), (3, 2, 0)):
        with pytest.raises(pdattn.PdattnError):
            pdattn.select_workspace_size(*bad)

    def call(**kw):
        a = pdattn.SelectArgs(P, P, P, P, P, P, 3, 4, 2, 64, 16, 40, 12, 8, 1, 2, P, n)
        for k, v in kw.items():
            setattr(a, k, v)
        return L.pdattn_select_pages(ctypes.byref(a), None)
    assert L.pdattn_select_pages(None, None) == pdattn.INVALID_ARG
    assert call(num_seqs=0) == pdattn.OK
    for kw in [{f: None} for f in ("q", "codes", "exponents", "block_table", "context_lens", "selected", "workspace")] + [
            dict(num_seqs=-1), dict(num_q_heads=5), dict(num_first=-1), dict(num_recent=0), dict(num_first=7), dict(num_selected=2),
            dict(num_first=2 ** 31 - 1, num_recent=2 ** 31 - 1), dict(max_blocks_per_seq=0), dict(num_blocks=0)]:
        assert call(**kw) == pdattn.INVALID_ARG, kw
    for kw in (dict(head_dim=96), dict(block_size=8), dict(num_q_heads=34)):
        assert call(**kw) == pdattn.UNSUPPORTED, kw
    assert call(q=P + 8) == call(codes=P + 8) == call(workspace=P + 128) == pdattn.MISALIGNED
    assert call(workspace_bytes=n - 1) == pdattn.WORKSPACE_TOO_SMALL


def test_selected_refusals():
    L = pdattn.lib()

    def both(sel=P, num=3, ks=P, vs=P, **kw):
        a = step(**kw)
        return (L.pdattn_decode_selected(ctypes.byref(a), sel, num, None), L.pdattn_decode_selected_fp8(ctypes.byref(a), sel, num, ks, vs, None))
    assert L.pdattn_decode_selected(None, P, 3, None) == L.pdattn_decode_selected_fp8(None, P, 3, P, P, None) == pdattn.INVALID_ARG
    assert both(num_seqs=0) == (pdattn.OK,) * 2
    for kw in (dict(sel=None), dict(num=0), dict(num=-1), dict(num=2 ** 31 - 1)):
        assert both(**kw) == (pdattn.INVALID_ARG,) * 2, kw
    assert both(ks=None)[1] == both(vs=None)[1] == pdattn.INVALID_ARG
    for kw, why in BAD_STEPS:
        assert both(**kw) == (why,) * 2, kw
    for kw, why in BAD_STRIDES:
        assert both(**kw)[0] == why, kw
    lens = (ctypes.c_int32 * 3)(10, 65, 3)                                       # a row of 64 tokens
    assert both(context_lens_host=ctypes.addressof(lens)) == (pdattn.INVALID_ARG,) * 2


def test_shares_of_the_tree_kernel(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    here, exe = os.path.dirname(os.path.abspath(__file__)), str(tmp_path / "tree_cut_check")
    subprocess.check_call([cxx, "-O2", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", pd_build.CSRC,
                           os.path.join(here, "c", "tree_cut_check.cpp"), "-o", exe])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and "tree_cut_check: ok" in out.stdout, out.stdout + out.stderr
