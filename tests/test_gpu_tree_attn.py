"""GPU: attention of drafted trees over the paged cache against the fp64 oracle.

Tolerance.  The output is rounded to bf16 once, half a step: 2^-8 of its value.  The
weights enter the products with V as bf16 numbers, half a step each, while their sum
takes the fp32 values: at most 2^-8 sum p |v| / sum p =: 2^-8 mag, of which the rounding
of the output adds 2^-8 again.  Scores and sums in fp32 add less than 2^-13 mag: a score
of D <= 128 products is off by at most 2^-17 of sum |q k| (below 2^10 scaled here for
all but the largest q, whose weights are one-hot), sums by 2^-20.
"""
import numpy as np
import pytest
import torch

from oracle import tree_ref
from paper_2507_08523_amd import ilpc

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm GPU (run with -m 'not gpu' on the CPU)")
    ilpc.load()
    yield
    torch.cuda.synchronize()


def random_tree(n, rng, branch=2):
    return [-1] + [int(rng.integers(max(0, (i - 1) // branch - 2), (i - 1) // branch + 1)) for i in range(1, n)]


def seen_of(parents):
    s = np.zeros((len(parents), len(parents)), bool)
    for i, line in enumerate(tree_ref.ancestors(parents)):
        s[i, line] = True
    return s


class Batch:
    """Requests of `before` keys and nodes whose masks are `seen` (bool [n, n] each), in permuted blocks of
    pools whose other slots hold NaN."""

    def __init__(self, before, seen, Hq=4, Hkv=2, D=128, std=1.0, seed=0, extra=0, spare_cols=0, fused=False,
                 words=None, blank=()):
        rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        self.before, self.seen, self.Hq, self.Hkv, self.D = list(before), seen, Hq, Hkv, D
        self.new = [len(s) for s in seen]
        lens, n = [p + k for p, k in zip(before, self.new)], sum(self.new)
        bf = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)  # noqa: E731
        nb = sum(-(-x // 16) for x in lens) + 3
        mb = max(max(-(-x // 16) for x in lens), 1) + spare_cols
        ids = rng.permutation(nb)
        self.kd, self.vd = [bf(x, Hkv, D) for x in lens], [bf(x, Hkv, D) for x in lens]
        for r, i in blank:  # nodes without K and V (no row sees them)
            self.kd[r][before[r] + i] = float("nan")
            self.vd[r][before[r] + i] = float("inf")
        q = (bf(n, Hq, D) * std).to(torch.bfloat16)
        kp, vp = torch.full((nb, Hkv, 16, D), float("nan")), torch.full((nb, Hkv, D, 16), float("nan"))
        bt, at = np.full((len(lens), mb), -1, np.int32), 0
        for r, x in enumerate(lens):
            m = -(-x // 16)
            bt[r, :m] = ids[at:at + m]
            at += m
            for j in range(m):
                a, b = 16 * j, min(16 * j + 16, x)
                kp[bt[r, j], :, :b - a] = self.kd[r][a:b].float().permute(1, 0, 2)
                vp[bt[r, j], :, :, :b - a] = self.vd[r][a:b].float().permute(1, 2, 0)
        w = words or max(1, -(-max(self.new) // 64))
        masks = np.zeros((n + extra, w, 64), np.uint64)
        row = 0
        for s in seen:
            k = len(s)
            masks[row:row + k].reshape(k, w * 64)[:, :k] = s
            row += k
        bits = (masks << np.arange(64, dtype=np.uint64)).sum(-1, dtype=np.uint64).view(np.int64)
        dev = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()  # noqa: E731
        self.kp, self.vp, self.masks = kp.to(torch.bfloat16).cuda(), vp.to(torch.bfloat16).cuda(), torch.from_numpy(bits).cuda()
        self.bt, self.cu, self.L = dev(bt), dev(np.concatenate([[0], np.cumsum(self.new)])), dev(lens)
        self.q = q.cuda()
        if fused:  # rows of a wider projection
            wide = torch.full((n, Hq + 2 * Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda")
            wide[:, :Hq] = self.q
            self.q = wide[:, :Hq]
        if extra:
            pad = torch.full((extra, *self.q.shape[1:]), float("nan"), dtype=torch.bfloat16, device="cuda")
            self.q = torch.cat([self.q, pad])
        self.scale, self.max_q = D ** -0.5, max(self.new)

    def run(self, out=None, max_q=None, **kw):
        out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
        ilpc.paged_tree_attn(self.q, self.kp, self.vp, self.bt, self.cu, self.L, max_q or self.max_q, self.scale,
                             self.masks, out, **kw)
        return out

    def check(self, out, rows_of=None):
        torch.cuda.synchronize()
        got, cu = out.float().cpu().numpy(), np.concatenate([[0], np.cumsum(self.new)])
        q = self.q.float().cpu().numpy()
        worst = 0.0
        for r, s in enumerate(self.seen):
            if not len(s) or (rows_of is not None and r not in rows_of):
                continue
            k, v = self.kd[r].float().numpy(), self.vd[r].float().numpy()
            k, v = np.where(np.isfinite(k), k, 0), np.where(np.isfinite(v), v, 0)
            ref, mag = tree_ref.tree_attention_ref(q[cu[r]:cu[r + 1]], k, v, self.scale, s)
            mine = got[cu[r]:cu[r + 1]]
            assert np.isfinite(mine).all(), f"request {r}"
            err, bound = np.abs(mine - ref), HALF * np.abs(ref) + (HALF * (1 + HALF) + 2.0 ** -13) * mag
            assert (err <= bound).all(), f"request {r}: {(err / np.maximum(bound, 1e-30)).max()}"
            worst = max(worst, float((err / np.maximum(bound, 1e-30)).max()))
        print(f"before {self.before[:4]} nodes {self.new[:4]} {self.Hq}/{self.Hkv}/{self.D}: {worst:.2f} of the bound",
              flush=True)


def trees(before, nodes, seed=0, **kw):
    rng = np.random.default_rng(seed)
    return Batch(before, [seen_of(random_tree(n, rng)) if n else np.zeros((0, 0), bool) for n in nodes], seed=seed, **kw)


HEADS = [(1, 1, 64), (4, 1, 64), (6, 2, 64), (8, 8, 128), (4, 2, 128), (7, 1, 128), (16, 2, 128), (20, 1, 64),
         (64, 1, 128)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("n", [1, 3, 13])
def test_head_shapes(heads, n):
    Hq, Hkv, D = heads
    b = trees([0, 3, 16, 31, 63, 64, 130], [n] * 7, seed=Hq, Hq=Hq, Hkv=Hkv, D=D)
    b.check(b.run())


@pytest.mark.parametrize("heads", HEADS)
def test_ragged_trees_over_ragged_contexts(heads):
    Hq, Hkv, D = heads
    b = trees([0, 1, 15, 17, 100, 129, 33], [5, 64, 0, 1, 33, 31, 90], seed=Hq, Hq=Hq, Hkv=Hkv, D=D)
    b.check(b.run())


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200])
@pytest.mark.parametrize("D", [64, 128])
def test_node_counts(n, D):
    # a request of n nodes beside one without any and one of a single node without context
    b = trees([48, 30, 0], [n, 0, 1], seed=n, Hq=4, Hkv=1, D=D)
    b.check(b.run())


@pytest.mark.parametrize("P", [0, 1, 2, 14, 15, 16, 17, 31, 32, 33, 63, 64, 65, 95, 127, 128, 500, 1023, 1024, 4000, 9001])
@pytest.mark.parametrize("n", [1, 20])
def test_context_lengths(P, n):
    # one request alone (its keys go over many workgroups), with spare table columns
    b = trees([P], [n], seed=P, Hq=8, Hkv=1, spare_cols=37)
    b.check(b.run())


@pytest.mark.parametrize("B", [1, 2, 5, 33, 70, 140, 300])
def test_batch_sizes(B):
    # the plan of waves and workgroups to a request changes with their number
    rng = np.random.default_rng(B)
    before = [int(x) for x in rng.integers(0, 700, B)]
    b = trees(before, [1] * B, seed=B, Hq=8, Hkv=8, D=64)
    b.check(b.run())
    nodes = [int(x) for x in rng.integers(0, 30, B)]
    nodes[0] = max(nodes[0], 1)
    b = trees(before, nodes, seed=B, Hq=8, Hkv=2)
    b.check(b.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tiles", [0.6, 1.2, 2.2, 3.2])
@pytest.mark.parametrize("longest", [40, 700])
def test_one_tile_of_columns_a_pair(D, tiles, longest):
    # by tiles of 32 columns to a compute unit
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    B = -(-int(tiles * cus) // 8)
    rng = np.random.default_rng(B)
    before = [longest] + [int(x) for x in rng.integers(0, longest + 1, B - 1)]
    b = trees(before, [8] + [int(x) for x in rng.integers(0, 9, B - 1)], seed=B, Hq=32, Hkv=8, D=D, fused=D == 64)
    b.check(b.run())


def wide(before, nodes, Hq, Hkv, D, two_groups):
    """The requests again and again, until the kernel for many columns takes the batch: more than two tiles of 32
    columns to a compute unit (and well more: 2.5, D 64 3.5); with one group of waves, or (contexts of more than 1 K keys,
    at most one tile of 128 columns to a unit) two."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    cols = max(nodes) * (Hq // Hkv)
    t32, t128 = -(-cols // 32), -(-cols // 128)
    assert t32 > 1
    need = (7 if D == 64 else 5) * cus // 2 + 1
    k = -(-need // (len(before) * Hkv * t32))
    if two_groups:
        assert k * len(before) * Hkv * t128 <= cus and max(before) >= 1000
    return dict(before=list(before) * k, nodes=list(nodes) * k, Hq=Hq, Hkv=Hkv, D=D)


@pytest.mark.parametrize("heads", [h for h in HEADS if h[0] // h[1] > 1])
def test_many_columns_head_shapes(heads):
    Hq, Hkv, D = heads
    b = trees(**wide([0, 3, 16, 31, 63, 64, 130], [33, 40, 1, 0, 64, 17, 50], Hq, Hkv, D, False), seed=Hq)
    b.check(b.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [17, 32, 33, 63, 64, 65, 130])
def test_many_columns_node_counts(n, D):
    b = trees(**wide([48, 0, 200, 61], [n, n, n, n], 8, 2, D, False), seed=n, fused=True)
    b.check(b.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [0, 1, 15, 16, 31, 33, 47, 48, 49, 63, 64, 65, 95, 96, 127, 128, 129, 1500])
def test_many_columns_context_lengths(P, D):
    b = trees(**wide([P], [33], 16, 4, D, False), seed=P, spare_cols=5)
    b.check(b.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("longest", [1000, 1063, 1064, 1130])
def test_two_groups_of_waves(D, longest):
    # contexts of one tile of keys to many, so that the second group has none, as many, or one tile fewer
    before = [longest, 0, 1, 40, 63, 64, 65, 100, 127, 128, 129, 191, 192, 193, 700]
    nodes = [64, 64, 63, 24, 1, 64, 63, 28, 64, 64, 0, 64, 5, 63, 64]
    b = trees(**wide(before, nodes, 32, 4, D, True), seed=longest, fused=True, extra=3)
    out = b.run()
    b.check(out)
    assert (out[-3:] == 7).all()


def test_many_long_trees():
    b = trees([700] * 12 + [100] * 4, [64] * 12 + [60, 1, 0, 64], seed=1, Hq=32, Hkv=4)
    b.check(b.run())


@pytest.mark.parametrize("n", [300, 1000, 1024])
def test_the_largest_trees(n):
    b = trees([50, 7], [n, 3], seed=n, Hq=2, Hkv=1, D=64)
    b.check(b.run())
    chain = Batch([33], [np.tril(np.ones((n, n), bool))], Hq=2, Hkv=1, seed=n)
    chain.check(chain.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [(4, 1), (16, 2), (40, 8), (256, 8)])
def test_any_mask_rows_without_a_key_among_them(D, heads):
    rng = np.random.default_rng(D)
    seen = [rng.random((n, n)) < p for n, p in ((40, 0.1), (70, 0.5), (9, 0.0), (33, 1.0), (128, 0.02))]
    seen[0][5] = seen[4][100] = False
    for before in ([0] * 5, [0, 20, 0, 5, 61]):
        b = Batch(before, seen, *heads, D=D, seed=D)
        out = b.run()
        b.check(out)
        if before[4] == 0:
            cu = np.concatenate([[0], np.cumsum(b.new)])
            assert (out[cu[0] + 5] == 0).all() and (out[cu[2]:cu[3]] == 0).all() and (out[cu[4] + 100] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("two_groups", [False, True])
def test_tiles_of_columns_whose_rows_see_few_nodes_or_none(D, two_groups):
    # 128 columns are 16 rows here: of a request's tiles some see nothing, some the first nodes, some late ones alone
    n = 160
    seen = np.zeros((n, n), bool)
    seen[40:70, :3] = seen[70:71, 64] = seen[71:100, 130:] = True
    seen[100:130] = np.tril(np.ones((n, n), bool))[100:130]
    seen[150:] = True
    shape = wide([0, 64, 1000 if two_groups else 700, 1], [n] * 4, 16, 2, D, two_groups)
    b = Batch(seen=[seen] * len(shape.pop("nodes")), seed=D, **shape)
    out = b.run()
    b.check(out)
    assert (out[:40] == 0).all() and (out[130:150] == 0).all()


@pytest.mark.parametrize("heads", [(4, 1, 64), (32, 2, 128), (512, 8, 64), (256, 8, 128)])
def test_nodes_that_no_row_sees_may_hold_anything(heads):
    rng = np.random.default_rng(3)
    seen = [seen_of(random_tree(n, rng)) for n in (20, 70, 140)]
    blank = [(0, 3), (0, 19), (1, 0), (1, 66), (2, 31), (2, 64), (2, 139)]
    for r, i in blank:
        seen[r][:, i] = False
    b = Batch([40, 0, 13], seen, *heads, blank=blank, seed=3)
    b.check(b.run())


@pytest.mark.parametrize("std", [128 ** -0.5, 1.0, 4.0, 30.0])
@pytest.mark.parametrize("Hq", [16, 512])
def test_small_and_large_scores(std, Hq):
    b = trees([700, 40, 5], [40, 40, 40], seed=4, Hq=Hq, Hkv=8, std=std)
    b.check(b.run())


@pytest.mark.parametrize("copies", [1, 330])
def test_a_maximum_that_keeps_rising(copies):
    # every 32 keys the scores rise by much more than the growth that is let pass
    b = trees([600], [20], seed=5, Hq=4, Hkv=1)
    b.kd[0][:] = (b.kd[0].float() * 0.01).to(torch.bfloat16)
    q = b.q.float().cpu()
    mean = q.mean((0, 1))
    for j in range(620):
        b.kd[0][j] = b.kd[0][j] + (mean / mean.norm() * (j / 620) * 200).to(torch.bfloat16)
    for j, blk in enumerate(b.bt[0].tolist()):
        if blk >= 0:
            a, e = 16 * j, min(16 * j + 16, 620)
            b.kp[blk, :, :e - a] = b.kd[0][a:e].permute(1, 0, 2).cuda()
    if copies > 1:  # (requests that share all their blocks)
        n = b.q.shape[0]
        for name in ("kd", "vd", "seen", "new", "before"):
            setattr(b, name, getattr(b, name) * copies)
        b.q, b.masks, b.bt, b.L = b.q.repeat(copies, 1, 1), b.masks.repeat(copies, 1), b.bt.repeat(copies, 1), b.L.repeat(copies)
        b.cu = torch.arange(copies + 1, dtype=torch.int32, device="cuda") * n
    b.check(b.run())


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("nodes", [[1, 2], [90, 65]])
def test_row_strides_and_rows_behind_the_last(fused, nodes):
    b = trees([50, 7], nodes, seed=6, Hq=8, Hkv=2, fused=fused, extra=5)
    out = b.run()
    b.check(out)
    assert (out[sum(nodes):] == 7).all()


def test_masks_wider_than_the_longest_tree_and_bits_of_nodes_that_are_not_there():
    b = trees([50, 7, 0], [20, 33, 1], seed=7, words=3)
    out = b.run()
    b.check(out)
    for r, (n, at) in enumerate(zip(b.new, b.cu.tolist())):
        rows = b.masks[at:at + n]
        rows[:, 0] |= -1 << n
        rows[:, 1:] = -1
    again = b.run()
    torch.cuda.synchronize()
    assert torch.equal(out, again)


def test_rows_past_max_q_len_and_bad_rows_are_left_alone():
    b = trees([50, 7, 90, 20], [20, 12, 6, 4], seed=8, Hq=8, Hkv=1)
    out = b.run(max_q=12)
    torch.cuda.synchronize()
    assert (out[12:20] == 7).all()
    full = b.run()
    torch.cuda.synchronize()
    b.check(full)
    b.check(torch.cat([out[:12], full[12:20], out[20:]]))
    # more nodes than keys, rows past the buffers
    for change in (lambda: b.L.__setitem__(1, 11), lambda: b.cu.__setitem__(4, 43)):
        L, cu = b.L.clone(), b.cu.clone()
        change()
        out = b.run()
        torch.cuda.synchronize()
        skipped = 1 if int(b.L[1]) == 11 else 3
        at = np.concatenate([[0], np.cumsum(b.new)])
        assert (out[at[skipped]:at[skipped + 1]] == 7).all()
        b.check(out, rows_of=[r for r in range(4) if r != skipped])
        b.L.copy_(L), b.cu.copy_(cu)


def test_bad_blocks_touch_no_other_request():
    b = trees([50, 70, 90], [20, 12, 6], seed=9, Hq=8, Hkv=1)
    b.bt[1, 0], b.bt[1, 2], b.bt[1, 4] = 1 << 30, -7, b.kp.shape[0]
    b.check(b.run(), rows_of=[0, 2])


def test_one_request_one_result_whatever_the_batch():
    # a request's rows are the same bits at any place of a batch of the same shape
    b = trees([300] * 6, [24] * 6, seed=10, Hq=8, Hkv=2)
    first = b.run()
    torch.cuda.synchronize()
    for _ in range(3):
        assert torch.equal(first, b.run())


def test_streams_workspaces_and_graphs():
    b, c = trees([2000], [40], seed=11, Hq=8, Hkv=2), trees([900, 31], [64, 9], seed=12, Hq=8, Hkv=2)
    want = [b.run(), c.run()]
    torch.cuda.synchronize()
    # two streams at once, own workspaces
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(w) for w in want]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for x, s, o in zip((b, c), streams, outs):
            x.run(o, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    # two captured graphs, replayed in turn with eager work between
    graphs, gout = [], [torch.zeros_like(w) for w in want]
    for x, o in zip((b, c), gout):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run(o)
        graphs.append(g)
    for k in range(4):
        for o in gout:
            o.zero_()
        b.q.mul_(1.0 if k % 2 else 0.5), c.q.mul_(1.0 if k % 2 else 0.5)
        for g in graphs:
            g.replay()
        eager = [b.run(), c.run()]
        torch.cuda.synchronize()
        assert torch.equal(gout[0], eager[0]) and torch.equal(gout[1], eager[1])


def test_the_binding_refuses():
    b = trees([50, 7], [20, 12], seed=13)
    out = torch.zeros_like(b.q)
    call = lambda **k: ilpc.paged_tree_attn(**dict(  # noqa: E731
        dict(q=b.q, k_pool=b.kp, v_pool=b.vp, block_tables=b.bt, cu_q=b.cu, seq_lens=b.L, max_q_len=20, scale=0.1,
             masks=b.masks, out=out), **k))
    call()
    for bad in (dict(masks=b.masks[:-1]), dict(masks=b.masks.int()), dict(masks=b.masks[:, 0]), dict(out=b.q),
                dict(out=out[:-1]), dict(seq_lens=b.L[:1]), dict(block_tables=b.bt[:1]), dict(q=b.q.float()),
                dict(max_q_len=65), dict(scale=-1.0), dict(scale=float("nan")), dict(v_pool=b.kp),
                dict(workspace=torch.zeros(4, device="cuda"))):
        with pytest.raises(ilpc.ILPCError):
            call(**bad)
    need = ilpc.tree_attn_workspace_bytes(2, 20, 4, 2, 128, b.bt.shape[1])
    if need:
        with pytest.raises(ilpc.ILPCError, match="workspace"):
            call(workspace=torch.zeros(need - 1, dtype=torch.uint8, device="cuda"))
    # keyword and integer-scale calls go the general way to the same kernels
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    want = b.run()
    call(scale=b.scale, workspace=ws, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def permuted(b, order):
    """The batch with its requests in another order: the same blocks, rows and masks."""
    c = object.__new__(Batch)
    c.__dict__.update(b.__dict__)
    at = np.concatenate([[0], np.cumsum(b.new)])
    rows = torch.from_numpy(np.concatenate([np.arange(at[r], at[r + 1]) for r in order])).cuda()
    idx = torch.tensor(order, device="cuda")
    c.q, c.masks = b.q[rows].contiguous(), b.masks[rows].contiguous()
    c.bt, c.L = b.bt[idx].contiguous(), b.L[idx].contiguous()
    c.new = [b.new[r] for r in order]
    c.cu = torch.tensor(np.concatenate([[0], np.cumsum(c.new)]), dtype=torch.int32, device="cuda")
    return c, rows


SHAPES = {  # kernel -> (tokens before, nodes) of the batch that it takes
    "stream": ([40, 0, 250, 7, 100, 31], [24, 3, 17, 0, 20, 24]),
    "stream and join": ([4000, 0, 2500, 700, 1, 3333], [24, 3, 17, 0, 20, 24]),
    "tiles": ([90, 0, 40, 64, 65], [33, 40, 1, 64, 17]),
    "tiles, two groups": ([1000, 0, 40, 700, 65], [33, 40, 1, 64, 17])}


def batch_of(kind, D, seed):
    before, nodes = SHAPES[kind]
    if "tiles" in kind:
        return trees(**wide(before, nodes, 32, 4, D, "two" in kind), seed=seed)
    return trees(before, nodes, seed=seed, Hq=8, Hkv=2, D=D)


@pytest.mark.parametrize("kind", list(SHAPES))
@pytest.mark.parametrize("D", [64, 128])
def test_a_requests_rows_are_the_same_bits_at_any_place_of_the_batch(kind, D):
    b = batch_of(kind, D, 14)
    need = ilpc.tree_attn_workspace_bytes(len(b.new), b.max_q, b.Hq, b.Hkv, D, b.bt.shape[1])
    assert (need > 0) == (kind == "stream and join")
    first = b.run()
    rng = np.random.default_rng(1)
    for _ in range(3):
        c, rows = permuted(b, rng.permutation(len(b.new)).tolist())
        out = c.run()
        torch.cuda.synchronize()
        assert torch.equal(out, first[rows])
    # other neighbours, of the same largest sizes
    n = b.new[0]
    b.q[n:] = (b.q[n:].flip(0) * 1.5).to(torch.bfloat16)
    b.bt[1:] = b.bt[1:].flip(0)
    again = b.run()
    torch.cuda.synchronize()
    assert torch.equal(again[:n], first[:n])
    b.check(first, rows_of=[0])
