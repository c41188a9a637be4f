"""Timed cases of the operators for growing batches on the GPU and for
differential attention, each with its plain form in elementary torch operations.

    extend    block tables, row offsets and slot map of a batch that grows by
              new tokens, its blocks taken from a free list on the device
    release   blocks of finished requests (or of tokens taken back) returned to it
    append    K/V rows stored into the paged pools through a slot map
    prefill   differential attention of packed suffix rows over the paged cache
    decode    the same of one to a few newest rows a request
    step      a whole decode step: extend, append, differential attention

Differential attention is the difference of two softmax maps over one set of
values: with the halves q = [q1 | q2], k = [k1 | k2] of a head of D dimensions
    y = (softmax(s q1 k1^T) - lambda_h softmax(s q2 k2^T)) V     (causal)
    out = out_scale * w * y / sqrt(mean(y^2) + eps)              (w: optional)
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BLOCK = 16
EPS = 1e-5

LLAMA, QWEN, LARGE, TINY = (32, 8, 128), (28, 4, 128), (64, 8, 128), (4, 1, 64)
# head shapes of the repository's workloads and of its shape tests
HEADS = [LLAMA, LLAMA, QWEN, LARGE, TINY, (8, 8, 128), (16, 2, 64), (20, 4, 128), (32, 2, 128), (12, 4, 64)]


def _case(kind, heads, b, shared, own_keys, new, name=None, q_std=1.0, norm=True, rope=False, fused=False, pad=0):
    """b requests of `shared` common tokens, then [lo, hi] of each one's own that
    the cache holds already, then [lo, hi] new ones; rope: halves in the pair
    layout; fused: q, k and v are views of one projection's output; pad: rows
    behind the last one."""
    hq, hkv, d = heads
    c = {"kind": kind, "hq": hq, "hkv": hkv, "d": d, "b": b, "shared": shared, "own_lo": own_keys[0],
         "own_hi": own_keys[1], "new_lo": new[0], "new_hi": new[1], "q_std": q_std, "norm": norm, "rope": rope,
         "fused": fused, "pad": pad}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the tables of a decode step of the largest batch: one token for each of 512 requests
        _case("extend", LARGE, 512, 0, (2000, 2140), (1, 1), "extend_decode"),
        # the tables of the largest prefill: 512 prompts of 1984 uncached tokens after a shared prefix
        _case("extend", LARGE, 512, 128, (0, 0), (1900, 1984), "extend_prefill"),
        # a few requests end
        _case("release", LLAMA, 4, 256, (300, 348), (1, 40), "release_few"),
        # a whole batch of long requests ends
        _case("release", LARGE, 512, 128, (0, 0), (1900, 1984), "release_batch"),
        # one new row of each of 512 requests, views of the layer's fused projection
        _case("append", LARGE, 512, 0, (2000, 2140), (1, 1), "append_decode", fused=True),
        # ragged suffixes of a serving step, half of each prompt cached
        _case("append", LLAMA, 64, 256, (0, 96), (200, 400), "append_prefill"),
        # the smallest batch of the repository: launches and latency only
        _case("prefill", TINY, 4, 64, (0, 0), (32, 32), "diff_prefill_tiny"),
        # a serving step: 64 prompts of about 600 tokens, half cached
        _case("prefill", LLAMA, 64, 256, (0, 96), (260, 300), "diff_prefill_serve", rope=True),
        # the largest heads and prompts, little cached
        _case("prefill", LARGE, 64, 128, (0, 0), (1900, 1984), "diff_prefill_large"),
        # decode of a handful of requests: each one's keys over many compute units
        _case("decode", LARGE, 4, 0, (2100, 2130), (1, 1), "diff_decode_few"),
        # decode of the largest batch, contexts of about 2.1 K tokens
        _case("decode", LARGE, 512, 0, (2100, 2140), (1, 1), "diff_decode_large"),
        # a decode step whose tables never leave the device, projections fused
        _case("step", LLAMA, 128, 512, (60, 540), (1, 1), "step_decode", fused=True, pad=32),
    ]


_MOST_FLOPS, _MOST_BYTES = 3.6e12, 4.2e9


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["extend", "release", "append", "prefill", "prefill", "decode", "decode", "step"])
        heads = rng.choice(HEADS)
        b = _log_int(rng, 1, 512)
        shared = rng.choice([0, BLOCK * _log_int(rng, 1, 96)])
        own_hi = rng.choice([0, _log_int(rng, 1, 4096)])
        own_keys = (rng.randint(own_hi // 2, own_hi), own_hi)
        if kind in ("decode", "step"):
            rows = rng.choice([1, 1, 1, 2, 3])
            new = (1, rows)
        else:
            hi = _log_int(rng, 1, 2112)
            new = (rng.randint(max(1, hi // 2), hi), hi)
        c = _case(kind, heads, b, shared, own_keys, new, None, rng.choice([heads[2] ** -0.5, 1.0, 1.0, 2.0]),
                  rng.random() < 0.7, rng.random() < 0.4, rng.random() < 0.4,
                  rng.choice([0, 0, _log_int(rng, 1, 64)]) if kind in ("extend", "append", "step") else 0)
        if kind in ("append", "prefill", "decode", "step") and c["b"] * (shared + own_hi + new[1]) > 1500000:
            continue
        w = work(c)
        if w["flops"] <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES:
            return c


# -- shapes -------------------------------------------------------------------

def _lens(case):
    """(tokens held, new tokens) of every request, the same for every seed."""
    b = case["b"]
    rng = np.random.default_rng([b, case["own_hi"], case["new_hi"]])

    def spread(lo, hi):
        return rng.permutation(np.round(np.linspace(lo, hi, b)).astype(np.int64))

    return case["shared"] + spread(case["own_lo"], case["own_hi"]), spread(case["new_lo"], case["new_hi"])


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    P, S = (x.astype(np.float64) for x in _lens(case))
    L, n, b = P + S, float(S.sum()), case["b"]
    kv, qo = 4.0 * case["hkv"] * case["d"], 2.0 * case["hq"] * case["d"]
    taken = float(np.sum(np.ceil(L / BLOCK) - np.ceil(P / BLOCK)))
    tables = 8.0 * b + 12.0 * b + 8.0 * taken + 4.0 * (n + case["pad"])
    append = (2 * kv + 4.0) * n
    pairs = float(np.sum(S * P + S * (S + 1) / 2))
    # the shared keys count once, a request's own once; Q in, output out
    whole = case["shared"] // BLOCK * BLOCK
    attn = kv * (float(np.sum(L - whole)) + whole) + 2 * qo * n
    # both maps' scores 2 D, the difference of the maps times V 2 D
    flops = 4.0 * case["hq"] * case["d"] * pairs
    kind = case["kind"]
    if kind == "extend":
        return {"bytes": tables, "flops": 0.0}
    if kind == "release":
        gone = float(np.sum(np.ceil(L / BLOCK) - case["shared"] // BLOCK))
        return {"bytes": 12.0 * b + 8.0 * gone, "flops": 0.0}
    if kind == "append":
        return {"bytes": append, "flops": 0.0}
    if kind == "step":
        return {"bytes": tables + append + attn, "flops": flops}
    return {"bytes": attn, "flops": flops}


# -- inputs -------------------------------------------------------------------

def prepare(case, seed):
    P, S = _lens(case)
    L = P + S
    b, hq, hkv, d, kind = case["b"], case["hq"], case["hkv"], case["d"], case["kind"]
    rng = np.random.default_rng([seed, 1])
    n = int(S.sum())
    rows = n + case["pad"]
    max_blocks = int(_blocks(L.max())) + 1
    # blocks: the shared ones, then every request's own, in a shuffled order; some to spare
    common = case["shared"] // BLOCK
    held = _blocks(P) if kind in ("extend", "step") else _blocks(L)
    need = int(np.sum(_blocks(L) - _blocks(P)))
    total = common + int(np.sum(held - common))
    num_blocks = total + need + 8
    perm = rng.permutation(num_blocks).astype(np.int32)
    tables = np.full((b, max_blocks), -1, np.int32)
    tables[:, :common] = perm[:common]
    at = common
    for r in range(b):
        k = int(held[r]) - common
        tables[r, common:common + k] = perm[at:at + k]
        at += k

    def dev(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    st = {"case": case, "num_blocks": num_blocks, "tables": dev(tables), "scale": (d // 2) ** -0.5}
    cu = np.concatenate([[0], np.cumsum(S)])
    if kind in ("extend", "step"):
        # the free list, some of whose head is taken already
        taken = 3
        ids = np.concatenate([np.arange(taken), perm[at:]])
        st.update(start=dev(P), new=dev(S), free=dev(ids), taken=dev([taken]), seq=dev(P * 0), cu=dev(cu * 0),
                  cu_blocks=dev(cu * 0), slots=dev(np.zeros(rows)), taken_out=dev([0]), status=dev([0]))
    if kind == "release":
        gone = int(np.sum(held - common))
        st.update(first=dev(np.full(b, common)), seq=dev(L), free=dev(np.concatenate([np.full(gone, -1), perm[at:]])),
                  taken=dev([gone]), cu_blocks=dev(cu * 0), taken_out=dev([0]), status=dev([0]))
    if kind in ("prefill", "decode"):
        st.update(seq=dev(L), cu=dev(cu))
    if kind == "append":
        pos = np.concatenate([np.arange(p, q) for p, q in zip(P, L)])
        req = np.repeat(np.arange(b), S)
        slots = np.full(rows, -1, np.int64)
        slots[:n] = tables[req, pos // BLOCK].astype(np.int64) * BLOCK + pos % BLOCK
        st["slots"] = dev(slots)
    if kind in ("extend", "release"):
        return st
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    st["k_pool"], st["v_pool"] = randn(num_blocks, hkv, BLOCK, d), randn(num_blocks, hkv, d, BLOCK)
    if case["fused"]:  # the layer's q, k and v come side by side
        x = randn(rows, hq + 2 * hkv, d)
        st["q"], st["k_new"], st["v_new"] = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    else:
        st["q"], st["k_new"], st["v_new"] = randn(rows, hq, d), randn(rows, hkv, d), randn(rows, hkv, d)
    if case["q_std"] != 1.0:
        st["q"].mul_(case["q_std"])
    st["max_q"] = int(S.max())
    st["out"] = torch.zeros(rows, hq, d, dtype=torch.bfloat16, device="cuda")
    st["lam"] = torch.rand(hq, generator=gen, device="cuda") * 0.8 + 0.1
    st["norm"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda") if case["norm"] else None
    st["out_scale"] = 0.2 if case["norm"] else 1.0
    return st


# -- one pass -----------------------------------------------------------------

def run(st):
    case, kind = st["case"], st["case"]["kind"]
    if own:
        return _run_own(st, kind)
    if kind == "extend":
        return _plain_extend(st)
    if kind == "release":
        return _plain_release(st)
    if kind == "append":
        _plain_append(st, st["slots"], case["pad"] > 0)
        return {"k_pool": st["k_pool"], "v_pool": st["v_pool"]}
    if kind == "step":
        res = _plain_extend(st)
        _plain_append(st, res["slot_map"], case["pad"] > 0)
        _plain_attn(st, res["block_tables"], res["seq_lens"])
        return {**res, "k_pool": st["k_pool"], "v_pool": st["v_pool"], "out": st["out"]}
    _plain_attn(st, st["tables"], st["seq"])
    return {"out": st["out"]}


def _run_own(st, kind):
    from paper_2507_08523_amd import ilpc

    case = st["case"]
    if kind in ("extend", "step"):
        ilpc.extend_tables(st["tables"], st["start"], st["new"], st["free"], st["taken"], st["seq"], st["cu"],
                           st["cu_blocks"], st["slots"], st["taken_out"], st["status"], st["num_blocks"])
    if kind == "release":
        ilpc.release_tables(st["tables"], st["first"], st["seq"], st["free"], st["taken"], st["cu_blocks"],
                            st["taken_out"], st["status"])
        return {"free_ids": st["free"], "cu_blocks": st["cu_blocks"], "taken": st["taken_out"],
                "status": st["status"]}
    if kind in ("append", "step"):
        ilpc.kv_append_slots(st["k_new"], st["v_new"], st["k_pool"], st["v_pool"], st["slots"])
    if kind in ("prefill", "decode", "step"):
        layout = ilpc.DIFF_ROPE if case["rope"] else ilpc.DIFF_HALVES
        ilpc.paged_diff_attn(st["q"], st["k_pool"], st["v_pool"], st["tables"], st["cu"], st["seq"], st["max_q"],
                             st["scale"], st["lam"], st["out"], norm_weight=st["norm"], norm_eps=EPS,
                             out_scale=st["out_scale"], layout=layout)
    res = {}
    if kind in ("extend", "step"):
        res.update(block_tables=st["tables"], seq_lens=st["seq"], cu_q=st["cu"], cu_blocks=st["cu_blocks"],
                   slot_map=st["slots"], taken=st["taken_out"], status=st["status"])
    if kind in ("append", "step"):
        res.update(k_pool=st["k_pool"], v_pool=st["v_pool"])
    if kind in ("prefill", "decode", "step"):
        res["out"] = st["out"]
    return res


# -- plain forms ----------------------------------------------------------------

def _sums(x):
    """0 and the running sums of x."""
    return torch.cat([x.new_zeros(1), torch.cumsum(x, 0)])


def _plain_extend(st):
    start, new, table = st["start"].long(), st["new"].long(), st["tables"]
    b, mb = table.shape
    rows, n_free = st["slots"].numel(), st["free"].numel()
    seq, have = start + new, (start + BLOCK - 1) // BLOCK
    need = (seq + BLOCK - 1) // BLOCK - have
    cu, cb, taken = _sums(new), _sums(need), st["taken"].long()
    status = ((taken + cb[-1] > n_free) * 1 + (seq.max() > mb * BLOCK) * 2 + (cu[-1] > rows) * 4
              + (torch.minimum(start, new).min() < 0) * 8)
    ok = status == 0
    j = torch.arange(mb, device="cuda")[None, :]
    fresh = (j >= have[:, None]) & (j < (have + need)[:, None]) & ok
    ids = st["free"][(taken + cb[:-1, None] + j - have[:, None]).clamp(0, n_free - 1)]
    st["tables"].copy_(torch.where(fresh, ids, table))
    i = torch.arange(rows, device="cuda")
    r = torch.searchsorted(cu[1:], i, right=True).clamp(max=b - 1)
    pos = start[r] + i - cu[r]
    phys = st["tables"][r, (pos // BLOCK).clamp(0, mb - 1)].long()
    slots = torch.where((i < cu[-1]) & ok & (phys >= 0) & (phys < st["num_blocks"]), phys * BLOCK + pos % BLOCK, -1)
    zero = cu.new_zeros(())
    return {"block_tables": st["tables"], "seq_lens": torch.where(ok, seq, start).int(),
            "cu_q": torch.where(ok, cu, zero).int(), "cu_blocks": torch.where(ok, cb, zero).int(),
            "slot_map": slots.int(), "taken": torch.where(ok, taken + cb[-1], taken).int(), "status": status.int()}


def _plain_release(st):
    first, table, taken = st["first"].long(), st["tables"], st["taken"].long()
    mb, n_free = table.shape[1], st["free"].numel()
    last = (st["seq"].long() + BLOCK - 1) // BLOCK
    count = (last - first).clamp(min=0)
    cb = _sums(count)
    status = (cb[-1] > taken) * 1 + (last.max() > mb) * 2 + (torch.minimum(first, st["seq"]).min() < 0) * 8
    ok = status == 0
    j = torch.arange(mb, device="cuda")[None, :]
    gone = (j >= first[:, None]) & (j < last[:, None]) & ok
    to = torch.where(gone, taken - cb[-1] + cb[:-1, None] + j - first[:, None], n_free)
    buf = torch.cat([st["free"], st["free"].new_zeros(1)])
    buf[to.reshape(-1)] = table.reshape(-1)
    st["free"].copy_(buf[:-1])
    zero = cb.new_zeros(())
    return {"free_ids": st["free"], "cu_blocks": torch.where(ok, cb, zero).int(),
            "taken": torch.where(ok, taken - cb[-1], taken).int(), "status": status.int()}


def _plain_append(st, slots, padded):
    k, v, s = st["k_new"], st["v_new"], slots.long()
    if padded:
        keep = s >= 0
        k, v, s = k[keep], v[keep], s[keep]
    st["k_pool"].permute(0, 2, 1, 3)[s // BLOCK, s % BLOCK] = k
    st["v_pool"].permute(0, 3, 1, 2)[s // BLOCK, s % BLOCK] = v


def _plain_attn(st, tables, seq_lens):
    """Requests in groups, padded to the group's longest: rows [g, Hkv, G * S, D]."""
    case = st["case"]
    hq, hkv, d, b = case["hq"], case["hkv"], case["d"], case["b"]
    g = hq // hkv
    P, S = _lens(case)
    cu = np.concatenate([[0], np.cumsum(S)])
    s_max, l_max = int(S.max()), int((P + S).max())
    per = max(1, min(b, int(6e8 / (hq * s_max * l_max)), int(1.2e9 / (hq * d * max(s_max, 1) + 2 * hkv * d * l_max))))
    n_blk = _blocks(l_max)
    key = torch.arange(l_max, device="cuda")
    m1 = _map_dims(case, 0)
    m2 = _map_dims(case, 1)
    lam = st["lam"].view(hkv, g, 1, 1)
    for r0 in range(0, b, per):
        r1 = min(b, r0 + per)
        nr = r1 - r0
        ids = tables[r0:r1, :n_blk].clamp(min=0).long()
        kk = st["k_pool"][ids].float().permute(0, 2, 1, 3, 4).reshape(nr, hkv, n_blk * BLOCK, d)[:, :, :l_max]
        vv = st["v_pool"][ids].float().permute(0, 2, 1, 4, 3).reshape(nr, hkv, n_blk * BLOCK, d)[:, :, :l_max]
        t = torch.arange(s_max, device="cuda")
        ln = seq_lens[r0:r1].long()
        n_new = torch.from_numpy(S[r0:r1]).cuda()
        row0 = torch.from_numpy(cu[r0:r1]).cuda()
        row = (row0[:, None] + torch.minimum(t[None, :], n_new[:, None] - 1))                 # [nr, s]
        pos = ln[:, None] - n_new[:, None] + torch.minimum(t[None, :], n_new[:, None] - 1)
        hidden = (key[None, None, :] > pos[:, :, None])[:, None, None]                        # [nr, 1, 1, s, l]
        qq = st["q"][row].float().view(nr, s_max, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(nr, hkv, g * s_max, d)
        vv = torch.where((key[None, :] < ln[:, None])[:, None, :, None], vv, 0.0).contiguous()
        a = None
        for dims in (m1, m2):
            kt = kk[..., dims].transpose(2, 3).contiguous()
            sc = torch.matmul(qq[..., dims].contiguous(), kt).mul_(st["scale"]).view(nr, hkv, g, s_max, l_max)
            sc.masked_fill_(hidden, -math.inf)
            sc.sub_(sc.amax(-1, keepdim=True)).exp_()
            sc.div_(sc.sum(-1, keepdim=True))
            a = sc if a is None else a.sub_(sc.mul_(lam))
            del sc
        y = torch.matmul(a.view(nr, hkv, g * s_max, l_max), vv).view(nr, hkv, g, s_max, d)
        del a
        if st["norm"] is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * st["norm"]
        y = (y * st["out_scale"]).permute(0, 3, 1, 2, 4).reshape(nr, s_max, hq, d).to(torch.bfloat16)
        if nr * s_max == cu[r1] - cu[r0]:
            st["out"][cu[r0]:cu[r1]] = y.reshape(-1, hq, d)
        else:
            st["out"][row] = y  # (a row behind a request's last repeats the last)


def _map_dims(case, m):
    """Dimensions of a head that map m reads: a half, or in the pair layout the
    dimensions i with i mod D/2 in the m-th half of D/2 (so that the rotation of
    pairs (i, i + D/2) stays within a map)."""
    i = torch.arange(case["d"])
    half = case["d"] // 2
    pick = i // half == m if not case["rope"] else (i % half) // (half // 2) == m
    return i[pick].cuda()


# -- the same in 64 bits --------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    kind, b = case["kind"], case["b"]
    P, S = _lens(case)
    L = P + S
    table = st["tables"].cpu().numpy().astype(np.int64)
    res = {}
    if kind in ("extend", "step"):
        free, at = st["free"].cpu().numpy(), int(st["taken"][0])
        cb, slots = [0], []
        for r in range(b):
            for j in range(int(_blocks(P[r])), int(_blocks(L[r]))):
                table[r, j] = free[at]
                at += 1
            cb.append(at - int(st["taken"][0]))
            pos = np.arange(P[r], L[r])
            slots.append(table[r, pos // BLOCK] * BLOCK + pos % BLOCK)
        slots.append(np.full(case["pad"], -1))
        res = {"block_tables": table, "seq_lens": L, "cu_q": np.concatenate([[0], np.cumsum(S)]),
               "cu_blocks": np.array(cb), "slot_map": np.concatenate(slots), "taken": np.array([at]),
               "status": np.array([0])}
        res = {k: torch.from_numpy(np.ascontiguousarray(v, dtype=np.int32)).cuda() for k, v in res.items()}
    if kind == "release":
        free, gone = st["free"].cpu().numpy().copy(), []
        cb = [0]
        for r in range(b):
            gone.extend(table[r, case["shared"] // BLOCK:int(_blocks(L[r]))])
            cb.append(len(gone))
        at = int(st["taken"][0])
        free[at - len(gone):at] = gone
        res = {"free_ids": free, "cu_blocks": np.array(cb), "taken": np.array([at - len(gone)]),
               "status": np.array([0])}
        return {k: torch.from_numpy(np.ascontiguousarray(v, dtype=np.int32)).cuda() for k, v in res.items()}
    if kind == "extend":
        return res
    tab = torch.from_numpy(table).cuda()
    if kind in ("append", "step"):
        # one request after the other, block by block positions
        row = 0
        for r in range(b):
            pos = torch.arange(int(P[r]), int(L[r]), device="cuda")
            phys, slot = tab[r][pos // BLOCK], pos % BLOCK
            rows = slice(row, row + int(S[r]))
            st["k_pool"][phys, :, slot] = st["k_new"][rows]
            st["v_pool"][phys, :, :, slot] = st["v_new"][rows]
            row += int(S[r])
        res.update(k_pool=st["k_pool"], v_pool=st["v_pool"])
    if kind == "append":
        return {k: x.double() for k, x in res.items()}
    if kind == "step":
        res.update(k_pool=st["k_pool"].double(), v_pool=st["v_pool"].double())
    res["out"] = _exact_attn(st, case, tab, P, S)
    return res


def _exact_attn(st, case, tab, P, S):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g, half = hq // hkv, d // 2
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lam = st["lam"].double()
    row = 0
    for r in range(case["b"]):
        p, s = int(P[r]), int(S[r])
        ln = p + s
        at = torch.arange(ln, device="cuda")
        phys, slot = tab[r][at // BLOCK], at % BLOCK
        seen = at[None, :] <= torch.arange(p, ln, device="cuda")[:, None]
        bias = torch.zeros(s, ln, dtype=torch.float64, device="cuda").masked_fill_(~seen, -math.inf)
        q = st["q"][row:row + s].double()
        k_all, v_all = st["k_pool"][phys, :, slot].double(), st["v_pool"][phys, :, :, slot].double()
        if case["rope"]:  # [a1 a2 b1 b2] -> [a1 b1 a2 b2]
            q = q.view(s, hq, 2, 2, half // 2).transpose(2, 3).reshape(s, hq, d)
            k_all = k_all.view(ln, hkv, 2, 2, half // 2).transpose(2, 3).reshape(ln, hkv, d)
        for h in range(hkv):
            qs = q[:, h * g:(h + 1) * g].transpose(0, 1).reshape(g * s, d)
            k, v = k_all[:, h], v_all[:, h]
            maps = []
            for m in (slice(0, half), slice(half, d)):
                z = torch.mm(qs[:, m].contiguous(), k[:, m].t().contiguous()).view(g, s, ln) * st["scale"] + bias
                maps.append(torch.softmax(z, dim=-1))
                del z
            diff = maps[0] - lam[h * g:(h + 1) * g, None, None] * maps[1]
            y = torch.mm(diff.view(g * s, ln), v).view(g, s, d)
            if st["norm"] is not None:
                y = y / torch.sqrt((y ** 2).mean(-1, keepdim=True) + EPS) * st["norm"].double()
            out[row:row + s, h * g:(h + 1) * g] = (y * st["out_scale"]).transpose(0, 1)
        row += s
    return out
