"""Refusals of the operators around the decode step, without a GPU: every bad argument is answered before any CUDA call."""
import ctypes

import pytest
import torch

from paper_2607_09207_b200 import build as pd_build
from paper_2607_09207_b200 import pdattn


@pytest.fixture(scope="module", autouse=True)
def _built():
    pd_build.build()


P = 0x10000      # an aligned address that no call may touch


def rope(**kw):
    a = pdattn.RopeArgs()
    for f in ("q", "q_out", "k_new", "v_new", "k_cache", "v_cache", "block_table", "context_lens", "cu_tokens", "inv_freq"):
        setattr(a, f, P)
    a.q_out = 2 * P
    a.q_token_stride, a.k_token_stride, a.v_token_stride = 256, 128, 128
    a.magnitude, a.rotary_dim, a.interleaved = 1.0, 64, 0
    a.num_tokens, a.num_seqs, a.num_q_heads, a.num_kv_heads, a.head_dim, a.block_size = 8, 3, 4, 2, 64, 16
    a.max_blocks_per_seq, a.num_blocks = 4, 12
    a.kv_block_stride, a.kv_head_stride, a.kv_token_stride = 2048, 1024, 64
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("fp8", [False, True])
def test_rope_append_refusals(fp8):
    L = pdattn.lib()

    def call(**kw):
        a = rope(**kw)
        return L.pdattn_rope_append_fp8(ctypes.byref(a), P, P, None) if fp8 else L.pdattn_rope_append(ctypes.byref(a), None)
    assert L.pdattn_rope_append(None, None) == pdattn.INVALID_ARG
    assert call(num_tokens=0) == pdattn.OK                                       # nothing to do
    for kw in (dict(num_tokens=-1), dict(num_seqs=0), dict(num_seqs=-1), dict(num_kv_heads=0), dict(num_q_heads=-1),
               dict(rotary_dim=0), dict(rotary_dim=80), dict(interleaved=2), dict(k_new=None), dict(v_new=None),
               dict(k_cache=None), dict(v_cache=None), dict(block_table=None), dict(context_lens=None), dict(inv_freq=None),
               dict(q=None), dict(q_out=None), dict(cu_tokens=None), dict(max_blocks_per_seq=0), dict(num_blocks=0),
               dict(q_token_stride=248), dict(k_token_stride=120), dict(v_token_stride=120),
               dict(q_out=P, q_token_stride=512)):
        assert call(**kw) == pdattn.INVALID_ARG, kw
    for kw in (dict(head_dim=96), dict(block_size=8), dict(rotary_dim=24), dict(q_token_stride=260), dict(k_token_stride=132)):
        assert call(**kw) == pdattn.UNSUPPORTED, kw
    for kw in (dict(q=P + 2), dict(q_out=P + 8), dict(k_new=P + 4), dict(v_new=P + 8), dict(k_cache=P + 8), dict(v_cache=P + 2)):
        assert call(**kw) == pdattn.MISALIGNED, kw
    if fp8:
        a = rope()
        assert L.pdattn_rope_append_fp8(ctypes.byref(a), None, P, None) == pdattn.INVALID_ARG
        assert L.pdattn_rope_append_fp8(ctypes.byref(a), P, None, None) == pdattn.INVALID_ARG
    else:
        assert call(kv_block_stride=0) == pdattn.INVALID_ARG and call(kv_token_stride=32) == pdattn.INVALID_ARG
        assert call(kv_head_stride=1028) == pdattn.UNSUPPORTED


def test_pages_refusals():
    L = pdattn.lib()
    n = pdattn.pages_workspace_size(12, 3)
    assert n % 256 == 0 and pdattn.pages_workspace_size(100000, 3) > n
    for bad in ((0, 3), (12, -1)):
        with pytest.raises(pdattn.PdattnError):
            pdattn.pages_workspace_size(*bad)
    good = pdattn.PoolArgs(P, P, P, 12)

    def calls(pool=good, table=P, lens=P, a=P, b=P, src=P, dst=P, S=3, MB=4, bs=16, n_fork=2, cap=6, ws=P, nb=n):
        p = ctypes.byref(pool) if pool is not None else None
        return [L.pdattn_pages_reserve(p, table, lens, a, S, MB, bs, ws, nb, None),
                L.pdattn_pages_fork(p, table, lens, a, b, n_fork, S, MB, bs, src, dst, ws, nb, None),
                L.pdattn_pages_free(p, table, lens, a, 2, S, MB, bs, ws, nb, None),
                L.pdattn_pages_compact(p, table, lens, S, MB, bs, src, dst, cap, ws, nb, None)]
    for kw in (dict(pool=None), dict(pool=pdattn.PoolArgs(None, P, P, 12)), dict(pool=pdattn.PoolArgs(P, None, P, 12)),
               dict(pool=pdattn.PoolArgs(P, P, None, 12)), dict(pool=pdattn.PoolArgs(P, P, P, 0)), dict(table=None),
               dict(lens=None), dict(S=-1), dict(MB=0), dict(bs=0), dict(ws=None)):
        assert calls(**kw) == [pdattn.INVALID_ARG] * 4, kw
    assert calls(bs=24) == [pdattn.UNSUPPORTED] * 4
    assert calls(ws=P + 64) == [pdattn.MISALIGNED] * 4
    assert calls(nb=n - 1) == [pdattn.WORKSPACE_TOO_SMALL] * 4
    assert calls(a=None)[:3] == [pdattn.INVALID_ARG] * 3
    assert calls(b=None)[1] == calls(src=None)[1] == calls(dst=None)[1] == calls(n_fork=4)[1] == calls(n_fork=-1)[1] == pdattn.INVALID_ARG
    assert calls(cap=5)[3] == calls(src=None)[3] == calls(dst=None)[3] == pdattn.INVALID_ARG
    assert L.pdattn_pages_reserve(ctypes.byref(good), None, None, None, 0, 4, 16, P, n, None) == pdattn.OK
    assert L.pdattn_pages_fork(ctypes.byref(good), P, P, None, None, 0, 3, 4, 16, None, None, P, n, None) == pdattn.OK
    assert L.pdattn_pages_init(None, None) == pdattn.INVALID_ARG

    def copy(k=P, v=P, src=P, dst=P, n=4, H=2, d=64, bs=16, NB=12, eb=2, sb=2048, sh=1024, st=64):
        return L.pdattn_pages_copy(k, v, src, dst, n, H, d, bs, NB, eb, sb, sh, st, None, None)
    assert copy(n=0) == pdattn.OK
    for kw in (dict(k=None), dict(v=None), dict(src=None), dict(dst=None), dict(n=-1), dict(H=0), dict(NB=0), dict(sb=0),
               dict(sh=-8), dict(st=56)):
        assert copy(**kw) == pdattn.INVALID_ARG, kw
    for kw in (dict(d=32), dict(bs=48), dict(eb=4), dict(sh=1028)):
        assert copy(**kw) == pdattn.UNSUPPORTED, kw
    assert copy(k=P + 8) == copy(v=P + 4) == pdattn.MISALIGNED


def test_status_strings_of_the_page_operations():
    L = pdattn.lib()
    assert len({L.pdattn_status_string(-i) for i in range(0, 11)}) == 11


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
             (dict(num_blocks=0), pdattn.INVALID_ARG), (dict(kv_head_stride=0), pdattn.INVALID_ARG), (dict(kv_token_stride=56), pdattn.INVALID_ARG),
             (dict(kv_block_stride=2052), pdattn.UNSUPPORTED), (dict(workspace=P + 128), pdattn.MISALIGNED),
             (dict(workspace_bytes=8447), pdattn.WORKSPACE_TOO_SMALL)]
BAD_STEPS += [({f: None}, pdattn.INVALID_ARG) for f in ("q", "k_cache", "v_cache", "out", "block_table", "context_lens", "workspace")]
BAD_STEPS += [({f: P + 8}, pdattn.MISALIGNED) for f in ("q", "k_cache", "v_cache", "out")]
BAD_SCORES = [(-1.0, 0), (float("nan"), 0), (float("inf"), 0), (0.0, -1)]


def test_prefill_refusals():
    L = pdattn.lib()

    def call(score=None, cu=P, n=9, **kw):
        return L.pdattn_prefill(ctypes.byref(step(**kw)), cu, n, None if score is None else ctypes.byref(score), None)
    assert L.pdattn_prefill(None, P, 9, None, None) == pdattn.INVALID_ARG
    assert call(n=0) == call(num_seqs=0) == pdattn.OK                            # nothing to do
    assert call(n=-1) == call(cu=None) == pdattn.INVALID_ARG
    for kw, why in BAD_STEPS:
        assert call(**kw) == why, kw
    for cap, window in BAD_SCORES:
        assert call(pdattn.ScoreArgs(cap, None, window, None, None, None)) == pdattn.INVALID_ARG
    assert pdattn.prefill_workspace_size(3, 9, 4, 2, 64) >= 8448
    with pytest.raises(pdattn.PdattnError):
        pdattn.prefill_workspace_size(3, -1, 4, 2, 64)


@pytest.mark.parametrize("fp8", [False, True])
def test_decode_scored_refusals(fp8):
    L = pdattn.lib()

    def call(score=pdattn.ScoreArgs(), **kw):
        a, s = ctypes.byref(step(**kw)), None if score is None else ctypes.byref(score)
        return L.pdattn_decode_scored_fp8(a, s, P, P, None) if fp8 else L.pdattn_decode_scored(a, s, None)
    assert call(score=None) == pdattn.INVALID_ARG
    assert call(num_seqs=0) == pdattn.OK
    for kw, why in BAD_STEPS:
        if not (fp8 and any("stride" in k for k in kw)):
            assert call(**kw) == why, kw
    for cap, window in BAD_SCORES:
        assert call(pdattn.ScoreArgs(cap, None, window, None, None, None)) == pdattn.INVALID_ARG
    lens = (ctypes.c_int32 * 3)(5, 6, 64)
    host = ctypes.cast(lens, ctypes.c_void_p).value
    assert call(pdattn.ScoreArgs(0.0, None, 0, P, None, None), context_lens_host=host) == pdattn.INVALID_ARG
    lens[2] = 65                                                                 # longer than its table row
    assert call(context_lens_host=host) == pdattn.INVALID_ARG
    if fp8:
        a, s = ctypes.byref(step()), ctypes.byref(pdattn.ScoreArgs())
        assert L.pdattn_decode_scored_fp8(a, s, None, P, None) == L.pdattn_decode_scored_fp8(a, s, P, None, None) == pdattn.INVALID_ARG


@pytest.mark.parametrize("cap", [1e-7, 1.5e6, 1e-44])
def test_caps_out_of_range(cap):
    L = pdattn.lib()
    score = ctypes.byref(pdattn.ScoreArgs(cap, None, 0, None, None, None))
    assert L.pdattn_prefill(ctypes.byref(step()), P, 9, score, None) == pdattn.INVALID_ARG
    assert L.pdattn_decode_scored(ctypes.byref(step()), score, None) == pdattn.INVALID_ARG
    assert L.pdattn_decode_scored_fp8(ctypes.byref(step()), score, P, P, None) == pdattn.INVALID_ARG


class Elsewhere:
    """Stands for a tensor of bytes on another device."""
    dtype, device, shape = torch.uint8, "cuda:7", (1 << 20,)

    def get_device(self):
        return 7

    def is_contiguous(self):
        return True

    def stride(self):
        return (1,)

    def numel(self):
        return 1 << 20

    def data_ptr(self):
        return P


def test_what_lives_on_another_device_is_refused_before_the_library_is_called(monkeypatch):
    """Host tensors take the part of the current device's."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)

    class Library:
        reached = 0

        def __getattr__(self, name):
            def call(*a):
                Library.reached += 1
                return pdattn.OK
            return call
    monkeypatch.setattr(pdattn, "_lib", Library())
    bf, i32 = torch.bfloat16, torch.int32
    q, kv, cache = torch.zeros(3, 4, 64, dtype=bf), torch.zeros(3, 2, 64, dtype=bf), torch.zeros(6, 2, 16, 64, dtype=bf)
    table, lens, cu = torch.zeros(3, 4, dtype=i32), torch.ones(3, dtype=i32), torch.arange(4, dtype=i32)
    freq, ws = torch.zeros(32), torch.zeros(1 << 16, dtype=torch.uint8)
    codes, scales = torch.zeros(6, 2, 16, 64, dtype=torch.uint8), torch.ones(2)
    vcodes = codes.transpose(2, 3).contiguous()
    pool = pdattn.PagePool(torch.zeros(6, dtype=i32), torch.zeros(6, dtype=i32), torch.zeros(1, dtype=i32))
    score = pdattn.Score(bias_slopes=torch.zeros(4))
    pairs = torch.zeros(3, dtype=i32)
    calls = {
        "rope": lambda w, s, p: pdattn.rope_append(q, kv, kv, q, cache, cache, table, lens, freq, workspace=w),
        "rope fp8": lambda w, s, p: pdattn.rope_append_fp8(q, kv, kv, q, codes, vcodes, scales, scales, table, lens, freq, workspace=w),
        "prefill": lambda w, s, p: pdattn.prefill(q, cache, cache, table, lens, cu, 1.0, q, w, score=s),
        "decode": lambda w, s, p: pdattn.decode_scored(q, cache, cache, table, lens, 1.0, q, w, s),
        "decode fp8": lambda w, s, p: pdattn.decode_scored_fp8(q, codes, vcodes, scales, scales, table, lens, 1.0, q, w, s),
        "reserve": lambda w, s, p: pdattn.pages_reserve(p, table, lens, lens, 16, w),
        "fork": lambda w, s, p: pdattn.pages_fork(p, table, lens, pairs, pairs, pairs, pairs, 16, w),
        "free": lambda w, s, p: pdattn.pages_free(p, table, lens, pairs, 16, w),
        "compact": lambda w, s, p: pdattn.pages_compact(p, table, lens, pairs, pairs, 16, w),
        "copy": lambda w, s, p: pdattn.pages_copy(cache, cache, pairs, pairs, workspace=w),
    }
    for name, call in calls.items():
        Library.reached = 0
        call(ws, score, pool)
        assert Library.reached == 1, name
        with pytest.raises(ValueError):
            call(Elsewhere(), score, pool)
        with pytest.raises(TypeError):
            call(ws.view(torch.int32), score, pool)
        with pytest.raises(ValueError):
            call(ws[:2], score, pool)
        assert Library.reached == 1, name
    monkeypatch.setattr(score, "device", 7)
    monkeypatch.setattr(pool, "device", 7)
    for name in ("prefill", "decode", "decode fp8", "reserve", "fork", "free", "compact"):
        with pytest.raises(ValueError):
            calls[name](ws, score, pool)
    assert Library.reached == 1


@pytest.mark.parametrize("off", [1, 2, 3])
def test_an_error_word_that_is_not_aligned_is_refused(off):
    """The kernels set bits of it atomically, so it has to be a whole word; any word will do."""
    L = pdattn.lib()
    ref = ctypes.byref

    def calls(ws):
        return [L.pdattn_rope_append(ref(rope(workspace=ws)), None), L.pdattn_rope_append_fp8(ref(rope(workspace=ws)), P, P, None),
                L.pdattn_pages_copy(P, P, P, P, 4, 2, 64, 16, 12, 2, 2048, 1024, 64, ws, None),
                L.pdattn_append_kv(P, P, P, P, P, P, 3, 2, 64, 16, 4, 12, 2048, 1024, 64, ws, None),
                L.pdattn_append_kv_fp8(P, P, P, P, P, P, P, P, 3, 2, 64, 16, 4, 12, ws, None)]
    assert calls(P + off) == [pdattn.MISALIGNED] * 5
    assert pdattn.MISALIGNED not in calls(P + 4 * off) if not torch.cuda.is_available() else True


def test_the_join_of_cut_prompt_items_stays_within_its_parts_whatever_the_workspace_holds(tmp_path):
    """The word that says how many parts an item has is not written when a call's waits run out."""
    import os
    import shutil
    import subprocess
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    here, exe = os.path.dirname(os.path.abspath(__file__)), str(tmp_path / "join_parts_check")
    subprocess.check_call([cxx, "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", pd_build.CSRC,
                           os.path.join(here, "c", "join_parts_check.cpp"), "-o", exe])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and "join_parts_check: ok" in out.stdout, out.stdout + out.stderr
    # and the kernel reads that word nowhere else
    with open(os.path.join(pd_build.CSRC, "prefill_umma.cuh")) as f:
        reads = [x for x in f.read().split("P.parts[item]")[1:] if not x.startswith(" = ")]
    assert len(reads) == 1 and reads[0].startswith(", P.splits);")


def test_a_scored_step_without_host_memory_for_its_plan_is_refused():
    """Not an exception through the C boundary, which would end the process.  In a child, whose address space is limited."""
    import subprocess
    import sys
    code = """
import ctypes, resource, sys
import numpy as np
lib = ctypes.CDLL(sys.argv[1])
sys.path.insert(0, sys.argv[2])
from paper_2607_09207_b200 import pdattn
n, P = 1 << 26, 0x10000
lens = np.ones(n, np.int32)
a = pdattn.Args()
for f in ("q", "k_cache", "v_cache", "out", "block_table", "context_lens", "workspace"):
    setattr(a, f, P)
a.context_lens_host = lens.ctypes.data
a.num_seqs, a.num_q_heads, a.num_kv_heads, a.head_dim, a.block_size = n, 4, 2, 64, 16
a.max_blocks_per_seq, a.num_blocks, a.scale = 4, 12, 0.1
a.kv_block_stride, a.kv_head_stride, a.kv_token_stride = 2048, 1024, 64
a.workspace_bytes = 1 << 62
s = pdattn.ScoreArgs(0.0, None, 5, None, None, None)
with open("/proc/self/statm") as f:
    used = int(f.read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (used + (64 << 20), resource.RLIM_INFINITY))
print("status", lib.pdattn_decode_scored(ctypes.byref(a), ctypes.byref(s), None))
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", code, pd_build.LIB, root], capture_output=True, text=True, timeout=300,
                         env=dict(os.environ, CUDA_VISIBLE_DEVICES=""))
    assert "status %d" % pdattn.UNSUPPORTED in out.stdout, out.stdout + out.stderr
