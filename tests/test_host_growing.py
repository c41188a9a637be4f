"""What the calls for growing batches and for differential attention refuse (CPU): every
argument is checked before anything is launched, in the library and in the binding."""
import ctypes

import pytest
import torch

from paper_2507_08523_amd import ilpc

P = 1 << 20  # stands for a device pointer in calls that are refused before it is used


def code(name, *args):
    return getattr(ilpc.load(), name)(*args)


def extend(**kw):
    a = dict(tables=P, mb=4, B=3, start=P, new=P, free=P, n_free=8, taken=P, nb=64, seq=P, cu=P, cb=P, slots=P,
             rows=8, out=P, status=P)
    assert not set(kw) - set(a)
    return code("ilpc_extend_tables", *dict(a, **kw).values(), None)


def release(**kw):
    a = dict(tables=P, mb=4, B=3, first=P, seq=P, free=P, n_free=8, taken=P, cb=P, out=P, status=P)
    assert not set(kw) - set(a)
    return code("ilpc_release_tables", *dict(a, **kw).values(), None)


def append(**kw):
    a = dict(k=P, ks=256, v=P, vs=256, kp=P, vp=P, nb=4, slots=P, n=3, Hkv=2, D=128, bs=16)
    assert not set(kw) - set(a)
    return code("ilpc_kv_append_slots", *dict(a, **kw).values(), None)


def attn(**kw):
    a = dict(q=P, qs=512, rows=3, kp=P, vp=P, nb=4, bt=P, mb=4, cu=P, L=P, B=2, mq=2, Hq=4, Hkv=2, D=128, bs=16,
             scale=0.1, layout=0, lam=P, w=P, eps=1e-5, out_scale=1.0, out=P, ws=None, wsb=0)
    assert not set(kw) - set(a)
    return code("ilpc_paged_diff_attn", *dict(a, **kw).values(), None)


@pytest.mark.parametrize("call,kw,rc", [
    *[(extend, {k: None}, ilpc.EINVAL) for k in ("tables", "start", "new", "free", "taken", "seq", "cu", "cb",
                                                 "slots", "out", "status")],
    *[(extend, {k: -1}, ilpc.EINVAL) for k in ("B", "n_free", "nb", "rows")], (extend, dict(mb=0), ilpc.EINVAL),
    (extend, dict(B=(1 << 20) + 1), ilpc.EUNSUP), (extend, dict(mb=(1 << 24) + 1), ilpc.EUNSUP),
    (extend, dict(nb=1 << 27), ilpc.EUNSUP),
    *[(release, {k: None}, ilpc.EINVAL) for k in ("tables", "first", "seq", "free", "taken", "cb", "out", "status")],
    (release, dict(B=-1), ilpc.EINVAL), (release, dict(n_free=-1), ilpc.EINVAL), (release, dict(mb=0), ilpc.EINVAL),
    (release, dict(B=(1 << 20) + 1), ilpc.EUNSUP), (release, dict(mb=(1 << 24) + 1), ilpc.EUNSUP),
    *[(append, {k: None}, ilpc.EINVAL) for k in ("k", "v", "kp", "vp", "slots")],
    *[(append, {k: P + 8}, ilpc.EINVAL) for k in ("k", "v", "kp", "vp")],
    *[(append, {k: s}, ilpc.EINVAL) for k in ("ks", "vs") for s in (248, 260)],
    (append, dict(n=-1), ilpc.EINVAL), (append, dict(Hkv=0), ilpc.EINVAL), (append, dict(D=96), ilpc.EUNSUP),
    (append, dict(bs=32), ilpc.EUNSUP), (append, dict(Hkv=65536, ks=1 << 23, vs=1 << 23), ilpc.EUNSUP),
    (append, dict(n=0, k=None, v=None), ilpc.OK),
    *[(attn, {k: None}, ilpc.EINVAL) for k in ("q", "kp", "vp", "bt", "cu", "L", "lam", "out")],
    *[(attn, {k: P + 8}, ilpc.EINVAL) for k in ("q", "kp", "vp", "w", "out")],
    *[(attn, {k: -1}, ilpc.EINVAL) for k in ("rows", "B", "mq", "nb")], (attn, dict(mb=0), ilpc.EINVAL),
    *[(attn, dict(qs=s), ilpc.EINVAL) for s in (508, 504)],
    *[(attn, dict(scale=s), ilpc.EINVAL) for s in (0.0, -0.1, float("inf"), float("nan"))],
    (attn, dict(out_scale=float("nan")), ilpc.EINVAL), (attn, dict(eps=-1e-5), ilpc.EINVAL),
    (attn, dict(eps=float("inf")), ilpc.EINVAL), (attn, dict(layout=2), ilpc.EINVAL),
    (attn, dict(D=32), ilpc.EUNSUP), (attn, dict(bs=8), ilpc.EUNSUP), (attn, dict(Hq=5), ilpc.EUNSUP),
    (attn, dict(Hq=130), ilpc.EUNSUP), (attn, dict(mb=(1 << 24) + 1), ilpc.EUNSUP),
    (attn, dict(B=1 << 30), ilpc.EUNSUP), (attn, dict(mq=1 << 30), ilpc.EUNSUP),
    (attn, dict(B=0, q=None), ilpc.OK), (attn, dict(mq=0, q=None), ilpc.OK), (attn, dict(rows=0, q=None), ilpc.OK),
])
def test_library_refuses_before_a_launch(call, kw, rc):
    assert call(**kw) == rc, ilpc.load().ilpc_last_error()


def test_workspace_size_refusals():
    n = ctypes.c_size_t()
    ref = ctypes.byref(n)
    assert code("ilpc_diff_attn_workspace_bytes", 2, 1, 4, 2, 128, 4, None) == ilpc.EINVAL
    for bad in ((-1, 1, 4, 2, 128, 4), (2, -1, 4, 2, 128, 4), (2, 1, 0, 2, 128, 4), (2, 1, 4, 2, 128, 0)):
        assert code("ilpc_diff_attn_workspace_bytes", *bad, ref) == ilpc.EINVAL
    for bad in ((2, 1, 5, 2, 128, 4), (2, 1, 4, 2, 80, 4), (1 << 30, 1, 4, 2, 128, 4)):
        assert code("ilpc_diff_attn_workspace_bytes", *bad, ref) == ilpc.EUNSUP
    n.value = 7
    assert code("ilpc_diff_attn_workspace_bytes", 0, 1, 4, 2, 128, 4, ref) == ilpc.OK and n.value == 0


def test_binding_takes_only_gpu_tensors():
    i, h, f = torch.zeros(3, dtype=torch.int32), torch.zeros(3, 2, 64).bfloat16(), torch.zeros(4)
    pool, pool_v = torch.zeros(4, 2, 16, 64).bfloat16(), torch.zeros(4, 2, 64, 16).bfloat16()
    bt, cu = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: ilpc.extend_tables(bt, i, i, i, i[:1], i, cu, cu, i, i[:1], i[:1], 4),
                 lambda: ilpc.release_tables(bt, i, i, i, i[:1], cu, i[:1], i[:1]),
                 lambda: ilpc.kv_append_slots(h, h, pool, pool_v, i),
                 lambda: ilpc.paged_diff_attn(h, pool, pool_v, bt, cu, i, 1, 0.1, f[:2], h.clone())):
        with pytest.raises(ilpc.ILPCError, match="must be a CUDA/HIP torch tensor"):
            call()


@pytest.mark.parametrize("call,kw,rc", [
    (append, dict(n=1 << 28), ilpc.EUNSUP),
    # the output on the queries' first row, on their last one (rows 512 elements apart), around them
    *[(attn, dict(out=P + x), ilpc.EINVAL) for x in (0, 2 * 2 * 512, -2 * 2 * 512)],
    (attn, dict(qs=2048, out=P + 2 * 512), ilpc.EINVAL),
])
def test_library_refuses_overlaps_and_grids_before_a_launch(call, kw, rc):
    assert call(**kw) == rc
    assert (b"overlap" if "out" in kw else b"too large") in ilpc.load().ilpc_last_error()


# (B, max_q_len, Hq, Hkv, D, max_blocks): what the documented limits allow, and not
ALLOWED = [(512, 131072, 64, 8, 128, 8192), (1 << 15, 1 << 19, 64, 8, 64, 9), (1 << 18, 1 << 16, 64, 1, 128, 4),
           (1 << 24, 1, 16, 1, 128, 4), (1 << 21, 1, 128, 8, 64, 9000), ((1 << 18) + 1, 63, 16, 1, 128, 4),
           (9, (1 << 16) + 1, 512, 8, 128, 4)]
TOO_LARGE = [(1 << 25, 1, 16, 1, 128, 9), (1 << 22, 1, 64, 8, 64, 9000), ((1 << 18) + 1, 128, 16, 1, 128, 9),
             (1 << 26, 1, 16, 1, 128, 4), (1 << 27, 1, 8, 1, 128, 4)]


def test_sizes_within_the_documented_limits_are_taken():
    n = ctypes.c_size_t()
    for sizes in ALLOWED:  # (EHIP: no device to ask)
        rc = code("ilpc_diff_attn_workspace_bytes", *sizes, ctypes.byref(n))
        assert rc in (ilpc.OK, ilpc.EHIP), (sizes, ilpc.load().ilpc_last_error())


@pytest.mark.parametrize("sizes", TOO_LARGE)
def test_query_and_launch_refuse_the_same_sizes(sizes):
    n = ctypes.c_size_t()
    B, mq, Hq, Hkv, D, mb = sizes
    assert code("ilpc_diff_attn_workspace_bytes", *sizes, ctypes.byref(n)) == ilpc.EUNSUP
    assert attn(B=B, mq=mq, Hq=Hq, Hkv=Hkv, D=D, mb=mb, qs=Hq * D, out=1 << 50) == ilpc.EUNSUP


def test_batches_past_both_grids_are_refused_before_a_launch():
    # more than 2^25 columns in all, most of the requests much shorter than the longest
    big = dict(B=1 << 15, mq=1 << 19, Hq=64, Hkv=8, D=64, mb=9, qs=4096, out=1 << 50)
    assert attn(rows=1 << 24, **big) == ilpc.EUNSUP
    assert b"too large" in ilpc.load().ilpc_last_error()


def test_the_committed_profile_names_the_current_kernel_code(monkeypatch):
    import os
    import re

    import bench

    text = open(os.path.join(bench.ROOT, "profiles", "diff_attn_kernel_trace.txt"), encoding="utf-8").read()
    found = dict(re.findall(r"^# code of (\w+\.hip): ([0-9a-f]{16})$", text, re.M))
    assert set(found) == {"diff_attn.hip", "diff_prefill.hip", "batch_tables.hip"}
    for name, sha in found.items():
        monkeypatch.setattr(bench, "KERNEL_SRC", os.path.join(bench.ROOT, "paper_2507_08523_amd", "csrc", name))
        assert bench.kernel_source_sha() == sha, name
