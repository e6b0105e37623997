"""Speculative decoding's entry points without a GPU: what they refuse before anything is enqueued, the
sizes they report, and that the binding's signatures are the header's.

As in test_abi.py, made-up device addresses are only handed over in a process that sees no CUDA
device; on a machine with a GPU this module re-runs itself in such a child."""
import ctypes
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_2409_04992_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000
E = binding
NEW = ["instinfer_tree_mask", "instinfer_decode_attention_tree", "instinfer_tree_workspace_bytes", "instinfer_verify_tree",
       "instinfer_kv_keep_path", "instinfer_kv_fork", "instinfer_kv_resize", "instinfer_kv_resize_workspace_bytes",
       "instinfer_kv_defragment", "instinfer_kv_defragment_workspace_bytes"]

fake_pointers = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: run in the GPU-less child instead")


@pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU here: the tests below run in this process")
def test_refusals_pass_in_a_child_that_sees_no_gpu():
    done = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-x", "-p", "no:cacheprovider"],
                          cwd=ROOT, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""), capture_output=True, text=True, timeout=600)
    assert done.returncode == 0, done.stdout[-3000:] + done.stderr[-2000:]
    assert " passed" in done.stdout


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def test_the_binding_has_the_headers_signatures(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "instinfer.h")).read(), flags=re.S)
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float, "size_t": ctypes.c_size_t}
    for name in NEW:
        found = re.search(r"(\w+)\s+%s\s*\((.*?)\);" % name, text, flags=re.S)
        want = [ctypes.c_void_p if "*" in p else kinds[p.split()[0]] for p in found.group(2).split(",")]
        function = getattr(lib, name)
        assert function.argtypes == want, name
        assert function.restype == (ctypes.c_size_t if found.group(1) == "size_t" else ctypes.c_int), name


def test_limits_are_the_headers():
    text = open(os.path.join(ROOT, "include", "instinfer.h")).read()
    value = lambda name: int(re.search(r"#define\s+%s\s+(\d+)" % name, text).group(1))  # noqa: E731
    assert (E.MAX_TREE_TOKENS, E.MAX_TREE_ROWS, E.MAX_LAYERS) == tuple(
        value("INSTINFER_" + n) for n in ("MAX_TREE_TOKENS", "MAX_TREE_ROWS", "MAX_LAYERS"))
    assert (E.FLAG_TREE_RANGE, E.FLAG_POOL) == (value("INSTINFER_FLAG_TREE_RANGE"), value("INSTINFER_FLAG_POOL"))


def tree(lib, **kw):
    a = dict(out=FAKE, lse=None, q=FAKE, k=FAKE, v=FAKE, table=None, lens=FAKE, trees=None, mask=FAKE, batch=2, nodes=8, hq=8,
             hkv=2, dim=128, s_max=256, T=0, M=0, P=0, max_len=256, scale=0.1, ws=FAKE, ws_bytes=1 << 34)
    a.update(kw)
    return lib.instinfer_decode_attention_tree(
        a["out"], a["lse"], a["q"], a["k"], a["v"], a["table"], a["lens"], a["trees"], a["mask"], a["batch"], a["nodes"], a["hq"],
        a["hkv"], a["dim"], a["s_max"], a["T"], a["M"], a["P"], a["max_len"], a["scale"], a["ws"], a["ws_bytes"], None, None)


@fake_pointers
def test_tree_attention_refuses(lib):
    for name in ("out", "q", "k", "v", "lens", "mask"):
        assert tree(lib, **{name: None}) == E.ERR_INVALID_ARG, name
    for name in ("out", "q", "k", "v", "mask"):
        assert tree(lib, **{name: FAKE + 8}) == E.ERR_INVALID_ARG, name
    for bad in (dict(batch=-1), dict(nodes=0), dict(hq=0), dict(hkv=0), dict(hq=7), dict(dim=0), dict(max_len=0), dict(s_max=0),
                dict(max_len=257), dict(scale=float("nan")), dict(scale=float("inf")), dict(table=FAKE, T=0, M=4, P=4),
                dict(table=FAKE, T=16, M=0, P=4), dict(table=FAKE, T=16, M=16, P=0), dict(table=FAKE, T=16, M=15, P=9)):
        assert tree(lib, **bad) == E.ERR_INVALID_ARG, bad
    for bad in (dict(dim=96), dict(nodes=129), dict(hq=2 * 65, nodes=64), dict(table=FAKE, T=8, M=32, P=9),
                dict(table=FAKE, T=24, M=32, P=9)):
        assert tree(lib, **bad) == E.ERR_UNSUPPORTED, bad
    for bad in (dict(ws=None), dict(ws=FAKE + 4), dict(ws_bytes=16),
                dict(ws_bytes=binding.tree_workspace_bytes(2, 8, 8, 2, 128, 256) - 1)):
        assert tree(lib, **bad) == E.ERR_WORKSPACE, bad
    assert tree(lib, batch=0, out=None, q=None) == E.OK
    for dim in (64, 128, 256):
        assert binding.tree_workspace_bytes(3, 64, 16, 4, dim, 5000) > 0
        assert binding.tree_workspace_bytes(0, 64, 16, 4, dim, 5000) > 0
    assert binding.tree_workspace_bytes(3, 64, 15, 4, 128, 5000) == 0
    assert binding.tree_workspace_bytes(3, 129, 16, 4, 128, 5000) == 0


@fake_pointers
def test_mask_and_verification_refuse(lib):
    def mask(out=FAKE, parents=FAKE, batch=2, nodes=8):
        return lib.instinfer_tree_mask(out, parents, None, batch, nodes, None, None)

    assert mask(out=None) == mask(out=FAKE + 8) == mask(parents=None) == mask(batch=-1) == mask(nodes=0) == E.ERR_INVALID_ARG
    assert mask(nodes=129) == E.ERR_UNSUPPORTED
    assert mask(batch=0, out=None) == E.OK

    def verify(**kw):
        a = dict(path=FAKE, lens=FAKE, out=FAKE, target=FAKE, draft=FAKE, kind=0, stride=100, tokens=FAKE, parents=FAKE, u=FAKE,
                 batch=2, nodes=8, vocab=100)
        a.update(kw)
        return lib.instinfer_verify_tree(a["path"], a["lens"], a["out"], a["target"], a["draft"], a["kind"], a["stride"],
                                         a["tokens"], a["parents"], None, a["u"], a["batch"], a["nodes"], a["vocab"], None, None)

    for name in ("path", "lens", "out", "target", "tokens", "parents", "u"):
        assert verify(**{name: None}) == E.ERR_INVALID_ARG, name
    for bad in (dict(target=FAKE + 4), dict(draft=FAKE + 2), dict(vocab=0), dict(stride=99), dict(batch=-1), dict(nodes=0),
                dict(vocab=(1 << 30) + 1, stride=1 << 40)):
        assert verify(**bad) == E.ERR_INVALID_ARG, bad
    assert verify(kind=3) == verify(kind=-1) == verify(nodes=129) == E.ERR_UNSUPPORTED
    assert verify(batch=0, path=None) == E.OK


def layers(*pointers):
    return (ctypes.c_void_p * len(pointers))(*pointers)


@fake_pointers
def test_keep_path_refuses(lib):
    def keep(**kw):
        a = dict(k=layers(FAKE, FAKE), v=layers(FAKE, FAKE), n=2, path=FAKE, lens=FAKE, seq=FAKE, new=2 * FAKE, table=None, M=0, T=0,
                 P=0, batch=2, nodes=8, heads=4, dim=128, s_max=64)
        a.update(kw)
        return lib.instinfer_kv_keep_path(a["k"], a["v"], a["n"], a["path"], a["lens"], None, a["seq"], a["new"], a["table"], a["M"],
                                          a["T"], a["P"], a["batch"], a["nodes"], a["heads"], a["dim"], a["s_max"], None, None)

    for bad in (dict(k=None), dict(v=None), dict(path=None), dict(lens=None), dict(seq=None), dict(new=None), dict(new=FAKE),
                dict(k=layers(FAKE, None)), dict(v=layers(FAKE, FAKE + 8)), dict(n=0), dict(heads=0), dict(dim=0), dict(s_max=0),
                dict(batch=-1), dict(nodes=0), dict(table=FAKE, M=4, T=16, P=0), dict(table=FAKE, M=0, T=16, P=4)):
        assert keep(**bad) == E.ERR_INVALID_ARG, bad
    for bad in (dict(n=129), dict(dim=96), dict(nodes=129), dict(table=FAKE, M=4, T=12, P=4)):
        assert keep(**bad) == E.ERR_UNSUPPORTED, bad
    assert keep(batch=0, k=None) == E.OK


@fake_pointers
def test_pool_calls_refuse(lib):
    def fork(**kw):
        a = dict(table=FAKE, refs=FAKE, seq=FAKE, src=FAKE, dst=FAKE, n=2, M=4, T=16, P=9, batch=3)
        a.update(kw)
        return lib.instinfer_kv_fork(a["table"], a["refs"], a["seq"], a["src"], a["dst"], a["n"], a["M"], a["T"], a["P"], a["batch"],
                                     None, None)

    def resize(**kw):
        a = dict(k=layers(FAKE), v=layers(FAKE), n=1, table=FAKE, refs=FAKE, seq=FAKE, want=FAKE, new=FAKE, M=4, T=16, P=9, batch=3,
                 heads=2, dim=128, ws=FAKE, ws_bytes=1 << 20)
        a.update(kw)
        return lib.instinfer_kv_resize(a["k"], a["v"], a["n"], a["table"], a["refs"], a["seq"], a["want"], a["new"], a["M"], a["T"],
                                       a["P"], a["batch"], a["heads"], a["dim"], a["ws"], a["ws_bytes"], None, None)

    def tidy(**kw):
        a = dict(k=layers(FAKE), v=layers(FAKE), n=1, table=FAKE, to=FAKE, refs=FAKE, new=FAKE, seq=FAKE, used=FAKE, M=4, T=16, P=9,
                 batch=3, heads=2, dim=128, ws=FAKE, ws_bytes=1 << 20)
        a.update(kw)
        return lib.instinfer_kv_defragment(a["k"], a["v"], a["n"], a["table"], a["to"], a["refs"], a["new"], a["seq"], a["used"],
                                           a["M"], a["T"], a["P"], a["batch"], a["heads"], a["dim"], a["ws"], a["ws_bytes"], None, None)

    pointers = {fork: ("table", "refs", "seq", "src", "dst"), resize: ("k", "v", "table", "refs", "seq", "want", "new"),
                tidy: ("k", "v", "table", "to", "refs", "new", "seq", "used")}
    for call, names in pointers.items():
        for name in names:
            assert call(**{name: None}) == E.ERR_INVALID_ARG, name
        for bad in (dict(M=0), dict(T=0), dict(P=0), dict(batch=-1), dict(P=1 << 31), dict(M=1 << 28)):
            assert call(**bad) == E.ERR_INVALID_ARG, bad
        for bad in (dict(T=12), dict(batch=8193), dict(batch=8192, M=1 << 16)):
            assert call(**bad) == E.ERR_UNSUPPORTED, bad
    assert fork(n=-1) == fork(n=4) == E.ERR_INVALID_ARG
    assert fork(n=0, src=None) == E.OK
    for call in (resize, tidy):
        for bad in (dict(n=0), dict(heads=0), dict(dim=0), dict(k=layers(FAKE + 8))):
            assert call(**bad) == E.ERR_INVALID_ARG, bad
        for bad in (dict(n=129), dict(dim=80)):
            assert call(**bad) == E.ERR_UNSUPPORTED, bad
        for bad in (dict(ws=None), dict(ws=FAKE + 8), dict(ws_bytes=64)):
            assert call(**bad) == E.ERR_WORKSPACE, bad
        assert call(batch=0, table=None) == E.OK
    assert binding.kv_resize_workspace_bytes(8193, 10) == 0 and binding.kv_resize_workspace_bytes(8192, 10) > 0
    assert binding.kv_defragment_workspace_bytes(0) == 0 and binding.kv_defragment_workspace_bytes(1 << 20) >= 8 << 20
