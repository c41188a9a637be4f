"""What the calls for drafted trees and forked rows refuse (CPU): every argument is checked
before anything is launched, in the library and in the binding."""
import ctypes
import os
import re
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2507_08523_amd import ilpc, pipeline

P = 1 << 20  # stands for a device pointer in calls that are refused before it is used


def code(name, *args):
    return getattr(ilpc.load(), name)(*args)


def caller(name, **defaults):
    def call(**kw):
        assert not set(kw) - set(defaults)
        return code(name, *dict(defaults, **kw).values(), None)
    call.__name__ = name
    return call


masks = caller("ilpc_tree_masks", par=P, cu=P, start=P, B=3, rows=9, words=1, masks=P, pos=P)
attn = caller("ilpc_paged_tree_attn", q=P, qs=512, rows=3, kp=P, vp=P, nb=4, bt=P, mb=4, cu=P, L=P, B=2, mq=2, Hq=4,
              Hkv=2, D=128, bs=16, scale=0.1, masks=P, words=1, out=P, ws=None, wsb=0)
accept = caller("ilpc_tree_accept", par=P, tok=P, pick=P, root=None, cu=P, start=P, B=3, rows=9, path=P, count=P,
                next=P, lens=P, blocks=P)
compact = caller("ilpc_kv_compact", kp=P, vp=P, nb=4, bt=P, mb=4, cu=P, start=P, B=3, rows=9, path=P, count=P, Hkv=2,
                 D=128, bs=16)
fork = caller("ilpc_fork_tables", bt=P, mb=4, B=3, seq=P, src=P, holds=P, first=2, free=P, n_free=8, taken=P, nb=64,
              cs=P, cd=P, out=P, status=P)
release = caller("ilpc_release_shared", bt=P, mb=4, B=3, seq=P, holds=P, first=2, free=P, n_free=8, taken=P, nb=64,
                 out=P, status=P)
copy = caller("ilpc_copy_blocks", kp=P, vp=P, nb=4, src=P, dst=P, n=3, Hkv=2, D=128, bs=16)

EINVAL, EUNSUP, OK = ilpc.EINVAL, ilpc.EUNSUP, ilpc.OK


@pytest.mark.parametrize("call,kw,rc", [
    *[(masks, {k: None}, EINVAL) for k in ("par", "cu", "masks")], (masks, dict(masks=P + 4), EINVAL),
    *[(masks, {k: -1}, EINVAL) for k in ("B", "rows")], (masks, dict(words=0), EINVAL), (masks, dict(words=17), EUNSUP),
    (masks, dict(B=(1 << 20) + 1), EUNSUP), (masks, dict(B=0, cu=None), OK), (masks, dict(rows=0, par=None), OK),
    *[(attn, {k: None}, EINVAL) for k in ("q", "kp", "vp", "bt", "cu", "L", "masks", "out")],
    *[(attn, {k: P + 8}, EINVAL) for k in ("q", "kp", "vp", "out")], (attn, dict(masks=P + 4), EINVAL),
    *[(attn, {k: -1}, EINVAL) for k in ("rows", "B", "mq", "nb")], (attn, dict(mb=0), EINVAL),
    (attn, dict(nb=0), EINVAL), *[(attn, dict(qs=s), EINVAL) for s in (508, 504)],
    *[(attn, dict(scale=s), EINVAL) for s in (0.0, -0.1, float("inf"), float("nan"))],
    (attn, dict(mq=65), EINVAL), (attn, dict(words=0), EINVAL), (attn, dict(words=17), EINVAL),
    (attn, dict(mq=1025, words=16), EUNSUP), (attn, dict(D=32), EUNSUP), (attn, dict(bs=8), EUNSUP),
    (attn, dict(Hq=5), EUNSUP), (attn, dict(Hq=130), EUNSUP), (attn, dict(mb=(1 << 24) + 1), EUNSUP),
    (attn, dict(B=1 << 30), EUNSUP), (attn, dict(B=(1 << 22) + 1), EUNSUP),
    # the output on the queries' first row, on their last one, around them
    *[(attn, dict(out=P + x), EINVAL) for x in (0, 2 * 2 * 512, -2 * 2 * 512)],
    (attn, dict(B=0, q=None), OK), (attn, dict(mq=0, q=None), OK), (attn, dict(rows=0, q=None), OK),
    *[(accept, {k: None}, EINVAL) for k in ("par", "tok", "pick", "cu", "start", "path", "count", "next", "lens",
                                            "blocks")],
    *[(accept, {k: -1}, EINVAL) for k in ("B", "rows")], (accept, dict(B=(1 << 20) + 1), EUNSUP),
    (accept, dict(B=0, cu=None), OK),
    *[(compact, {k: None}, EINVAL) for k in ("kp", "vp", "bt", "cu", "start", "path", "count")],
    *[(compact, {k: P + 8}, EINVAL) for k in ("kp", "vp")], *[(compact, {k: -1}, EINVAL) for k in ("B", "rows", "nb")],
    (compact, dict(mb=0), EINVAL), (compact, dict(Hkv=0), EINVAL), (compact, dict(D=96), EUNSUP),
    (compact, dict(bs=32), EUNSUP), (compact, dict(Hkv=65536), EUNSUP), (compact, dict(B=(1 << 20) + 1), EUNSUP),
    (compact, dict(mb=(1 << 24) + 1), EUNSUP), (compact, dict(B=0, kp=None), OK), (compact, dict(rows=0, path=None), OK),
    *[(fork, {k: None}, EINVAL) for k in ("bt", "seq", "src", "holds", "free", "taken", "cs", "cd", "out", "status")],
    *[(fork, {k: -1}, EINVAL) for k in ("B", "n_free", "nb", "first")], (fork, dict(mb=0), EINVAL),
    (fork, dict(first=65), EINVAL), (fork, dict(B=(1 << 20) + 1), EUNSUP), (fork, dict(mb=(1 << 24) + 1), EUNSUP),
    (fork, dict(nb=1 << 27), EUNSUP),
    *[(release, {k: None}, EINVAL) for k in ("bt", "seq", "holds", "free", "taken", "out", "status")],
    *[(release, {k: -1}, EINVAL) for k in ("B", "n_free", "nb", "first")], (release, dict(mb=0), EINVAL),
    (release, dict(first=65), EINVAL), (release, dict(B=(1 << 20) + 1), EUNSUP),
    (release, dict(mb=(1 << 24) + 1), EUNSUP), (release, dict(nb=1 << 27), EUNSUP),
    *[(copy, {k: None}, EINVAL) for k in ("kp", "vp", "src", "dst")], *[(copy, {k: P + 8}, EINVAL) for k in ("kp", "vp")],
    *[(copy, {k: -1}, EINVAL) for k in ("n", "nb")], (copy, dict(Hkv=0), EINVAL), (copy, dict(D=96), EUNSUP),
    (copy, dict(bs=8), EUNSUP), (copy, dict(Hkv=65536), EUNSUP), (copy, dict(n=1 << 23), EUNSUP),
    (copy, dict(n=0, src=None), OK),
])
def test_library_refuses_before_a_launch(call, kw, rc):
    assert call(**kw) == rc, ilpc.load().ilpc_last_error()


def test_size_queries():
    n, w = ctypes.c_size_t(), ctypes.c_int32()
    ref = ctypes.byref(n)
    assert code("ilpc_tree_attn_workspace_bytes", 2, 1, 4, 2, 128, 4, None) == EINVAL
    for bad in ((-1, 1, 4, 2, 128, 4), (2, -1, 4, 2, 128, 4), (2, 1, 0, 2, 128, 4), (2, 1, 4, 2, 128, 0)):
        assert code("ilpc_tree_attn_workspace_bytes", *bad, ref) == EINVAL
    for bad in ((2, 1, 5, 2, 128, 4), (2, 1, 4, 2, 80, 4), (1 << 30, 1, 4, 2, 128, 4), (2, 1025, 4, 2, 128, 4)):
        assert code("ilpc_tree_attn_workspace_bytes", *bad, ref) == EUNSUP
    n.value = 7
    assert code("ilpc_tree_attn_workspace_bytes", 0, 1, 4, 2, 128, 4, ref) == OK and n.value == 0
    for blocks, words in ((0, 0), (1, 2), (32, 33), (33, 35), (1000, 1032)):
        assert code("ilpc_holds_words", blocks, ctypes.byref(w)) == OK and w.value == words
        assert ilpc.holds_words(blocks) == words
    assert code("ilpc_holds_words", -1, ctypes.byref(w)) == EINVAL and code("ilpc_holds_words", 1, None) == EINVAL
    assert code("ilpc_holds_words", 1 << 27, ctypes.byref(w)) == EUNSUP


def test_binding_takes_only_gpu_tensors():
    i, i1, m = torch.zeros(3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(3, 1).long()
    h, cu, bt = torch.zeros(3, 2, 64).bfloat16(), torch.zeros(4, dtype=torch.int32), torch.zeros(3, 4, dtype=torch.int32)
    pool, pool_v = torch.zeros(4, 2, 16, 64).bfloat16(), torch.zeros(4, 2, 64, 16).bfloat16()
    holds = torch.zeros(5, dtype=torch.int32)
    for call in (lambda: ilpc.tree_masks(i, cu, m),
                 lambda: ilpc.paged_tree_attn(h, pool, pool_v, bt, cu, i, 1, 0.1, m, h.clone()),
                 lambda: ilpc.tree_accept(i, i, i, cu, i, i, i, i, i, i),
                 lambda: ilpc.kv_compact(pool, pool_v, bt, cu, i, i, i),
                 lambda: ilpc.fork_tables(bt, i, i, holds, 0, i, i1, i, i, i1, i1, 4),
                 lambda: ilpc.release_shared(bt, i, holds, 0, i, i1, i1, i1, 4),
                 lambda: ilpc.copy_blocks(pool, pool_v, i, i)):
        with pytest.raises(ilpc.ILPCError, match="must be a CUDA/HIP torch tensor"):
            call()


def test_the_committed_profile_names_the_current_kernel_code(monkeypatch):
    import bench

    with open(os.path.join(bench.ROOT, "profiles", "tree_attn_kernel_trace.txt"), encoding="utf-8") as f:
        named = dict(re.findall(r"^# code of (\w+\.hip): ([0-9a-f]{16})$", f.read(), re.M))
    assert sorted(named) == ["cache_forks.hip", "tree_attn.hip", "tree_draft.hip", "tree_tiles.hip"]
    for name, sha in named.items():
        monkeypatch.setattr(bench, "KERNEL_SRC", os.path.join(bench.ROOT, "paper_2507_08523_amd", "csrc", name))
        assert bench.kernel_source_sha() == sha, name


@pytest.mark.parametrize("n", [1025, 4096])
def test_tables_refuse_longer_drafts_than_the_calls_take(n):
    pc = SimpleNamespace(max_blocks=4)  # (refused before anything of it is used)
    with pytest.raises(ilpc.ILPCError, match="max_nodes") as e:
        pipeline.DeviceTables(pc, np.full((2, 4), -1, np.int32), [0, 0], 8, max_nodes=n)
    assert e.value.code == ilpc.EUNSUP


def test_the_committed_profile_names_the_headers_code(monkeypatch):
    # (tree_attn.h has the mask window, diff_attn.h the operand layouts)
    import bench

    with open(os.path.join(bench.ROOT, "profiles", "tree_attn_kernel_trace.txt"), encoding="utf-8") as f:
        named = dict(re.findall(r"^# code of (\w+\.h): ([0-9a-f]{16})$", f.read(), re.M))
    assert sorted(named) == ["diff_attn.h", "tree_attn.h"]
    for name, sha in named.items():
        monkeypatch.setattr(bench, "KERNEL_SRC", os.path.join(bench.ROOT, "paper_2507_08523_amd", "csrc", name))
        assert bench.kernel_source_sha() == sha, name


fork_drafts = caller("ilpc_fork_tables_drafts", bt=P, mb=4, B=3, seq=P, src=P, holds=P, first=2, free=P, n_free=8, taken=P,
                     nb=64, cs=P, cd=P, start=P, out=P, status=P)


@pytest.mark.parametrize("kw,rc", [
    *[({k: None}, EINVAL) for k in ("bt", "seq", "src", "holds", "free", "taken", "cs", "cd", "out", "status")],
    *[({k: -1}, EINVAL) for k in ("B", "n_free", "nb", "first")], (dict(mb=0), EINVAL), (dict(first=65), EINVAL),
    (dict(B=(1 << 20) + 1), EUNSUP), (dict(mb=(1 << 24) + 1), EUNSUP), (dict(nb=1 << 27), EUNSUP),
    (dict(start=None, B=(1 << 20) + 1), EUNSUP)])
def test_forks_beside_drafts_are_refused_alike(kw, rc):
    assert fork_drafts(**kw) == rc, ilpc.load().ilpc_last_error()
