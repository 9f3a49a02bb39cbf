"""hf_attend against the 64-bit form: types, head layouts, lengths from nothing
to many tiles, masks that leave rows empty, paged and strided caches, what lies
past the end, splits, offsets past 32 bits, streams and graphs."""

import numpy as np
import pytest
import torch

import cache_plain as P
from paper_2609_32259_gb300 import binding as B
from paper_2609_32259_gb300 import pipeline

pytestmark = pytest.mark.gpu

TDT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as g

    g.build()


def _i32(v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda")


def _ptr(lens):
    return _i32(np.concatenate([[0], np.cumsum(lens)]))


class Setup:
    """A cache with random rows for sequences of (queries, cache rows), everything
    that no sequence holds filled with NaN."""

    def __init__(self, kind, H, G, D, lens, block=0, seed=0, dtype=None, spare=2):
        self.kind, self.H, self.G, self.D, self.lens = kind, H, G, D, lens
        self.dtype = TDT[dtype or ("f32" if kind == "f32" else "bf16")]
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = len(lens)
        kv = [m for _, m in lens]
        if block:
            need = [-(-m // block) for m in kv]
            n_blocks = sum(need) + spare
            perm = torch.randperm(n_blocks, generator=g, device="cuda").to(torch.int32)
            mb = max(max(need), 1)
            self.table = torch.full((n, mb), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
            at = 0
            for i, c in enumerate(need):
                self.table[i, :c] = perm[at:at + c]
                at += c
            rows = n_blocks * block
            self.rows_of = [torch.cat([self.table[i].long()[:, None] * block + torch.arange(block, device="cuda")])
                            .reshape(-1)[:m] for i, m in enumerate(kv)]
            self.row0 = None
        else:
            self.table = None
            starts = np.cumsum([0] + [m + spare for m in kv])
            rows = int(starts[-1])
            self.row0 = _i32(starts[:-1])
            self.rows_of = [torch.arange(int(starts[i]), int(starts[i]) + m, device="cuda") for i, m in enumerate(kv)]
        used = torch.cat(self.rows_of) if n else torch.zeros(0, dtype=torch.long, device="cuda")
        if kind == "q4":
            x = torch.randn((2, rows, H, D), generator=g, device="cuda").cpu().numpy()
            val, codes, s = P.held_in_4_bits(x)
            codes = torch.as_tensor(P.pack_codes(codes)).cuda().permute(0, 2, 1, 3).contiguous()
            s = torch.as_tensor(s).cuda().permute(0, 2, 1, 3).contiguous().to(torch.bfloat16)
            free = torch.ones(rows, dtype=torch.bool, device="cuda")
            free[used] = False
            s[:, :, free] = float("nan")
            codes[:, :, free] = 0
            self.val = torch.as_tensor(val).cuda()
            self.cache = pipeline.KVCache(kind="q4", H=H, D=D, n_seq=n, codes=codes[None], scales=s[None],
                                          block_table=self.table, block_size=block, row0=self.row0)
        else:
            t = TDT[kind]
            kvt = torch.full((2, rows, H, D), float("nan"), dtype=t, device="cuda")
            kvt[:, used] = torch.randn((2, len(used), H, D), generator=g, device="cuda").to(t)
            self.val = kvt
            self.cache = pipeline.KVCache(kind=kind, H=H, D=D, n_seq=n, kv=kvt[None], block_table=self.table,
                                          block_size=block, row0=self.row0)
        self.q_ptr = _ptr([a for a, _ in lens])
        self.kv_len = _i32(kv)
        T = sum(a for a, _ in lens)
        self.q = (torch.randn((T, H * G, D), generator=g, device="cuda") * 1.5).to(self.dtype)

    def run(self, causal=True, scale=0.0, lse=True, q=None, out=None, hints=True, stream=None):
        q = self.q if q is None else q
        out = torch.full_like(q, float("nan")) if out is None else out
        e = torch.full(q.shape[:2], float("nan"), device="cuda") if lse else None
        kw = {}
        if hints:
            kw = dict(max_q_len=max(a for a, _ in self.lens), max_kv_len=max(m for _, m in self.lens))
        self.cache.attend(0, q, out, self.q_ptr, self.kv_len, causal=causal, scale=scale, lse=e, stream=stream, **kw)
        torch.cuda.synchronize()
        return out, e

    def check(self, out, lse, causal=True, scale=None):
        at = 0
        for (n, m), rows in zip(self.lens, self.rows_of):
            o, e, absv, size = P.attend(self.q[at:at + n], self.val[0, rows], self.val[1, rows], causal, scale)
            got = out[at:at + n].double()
            assert torch.isfinite(got).all()
            tol = P.bound(o, absv, size, self.dtype)
            bad = (got - o).abs() > tol
            assert not bad.any(), (n, m, ((got - o).abs() / tol).max().item(), int(bad.sum()), bad.nonzero()[:3].tolist())
            if lse is not None:
                gl = lse[at:at + n].double()
                assert torch.equal(torch.isinf(e), torch.isinf(gl))
                f = torch.isfinite(e)
                # scores as in bound(); their logarithm's own rounding
                assert ((gl - e).abs()[f] <= (2.0 ** -15 * (1 + size))[f] + 2.0 ** -22 * e.abs()[f]).all()
            at += n
        assert self.cache.status() == 0
        assert self.cache._workspace[:B.ATTEND_ZEROED].count_nonzero() == 0


RAGGED = [(1, 1), (0, 5), (3, 0), (5, 5), (17, 40), (130, 129), (64, 300)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,H,G,D", [
    ("f32", 4, 2, 32), ("f32", 1, 3, 96), ("f32", 2, 1, 128), ("f32", 1, 2, 256), ("bf16", 2, 2, 32),
    ("bf16", 1, 5, 96), ("bf16", 2, 4, 64), ("bf16", 2, 7, 128), ("bf16", 8, 1, 128), ("bf16", 1, 16, 128),
    ("bf16", 1, 2, 256), ("q4", 2, 4, 64), ("q4", 2, 7, 128), ("q4", 1, 3, 256),
])
def test_attend_ragged(kind, H, G, D, causal):
    # rows that see nothing, sequences without tokens or rows, tiles that end anywhere
    s = Setup(kind, H, G, D, RAGGED, block=16, seed=H * D + G)
    s.check(*s.run(causal), causal)


@pytest.mark.parametrize("kind,dtype", [("bf16", None), ("f32", None), ("q4", None), ("q4", "f32")])
@pytest.mark.parametrize("block", [0, 1, 8, 24, 64, 256])
def test_attend_layouts(kind, dtype, block):
    s = Setup(kind, 2, 4, 64, [(9, 200), (1, 77), (40, 40)], block=block, seed=block, dtype=dtype)
    s.check(*s.run())


@pytest.mark.parametrize("kind", ["bf16", "q4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 4097])
def test_attend_single_tokens(kind, D, m):
    s = Setup(kind, 2, 4, D, [(1, m), (1, max(1, m // 3)), (1, 1)], block=16, seed=m)
    s.check(*s.run())


@pytest.mark.parametrize("kind", ["bf16", "q4"])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8, 9, 12, 16, 17, 32, 64])
def test_attend_groups_of_heads(kind, G):
    s = Setup(kind, 1, G, 128, [(1, 300), (2, 33), (1, 0), (3, 2)], block=16, seed=G)
    s.check(*s.run())


@pytest.mark.parametrize("kind", ["bf16", "q4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,m", [(127, 127), (128, 128), (129, 129), (255, 300), (256, 256), (257, 513), (64, 1500),
                                 (1025, 1025), (31, 4000), (300, 100)])
def test_attend_prompts(kind, D, n, m):
    s = Setup(kind, 2, 3, D, [(n, m)], seed=n + m)
    s.check(*s.run())


@pytest.mark.parametrize("kind", ["bf16", "q4"])
@pytest.mark.parametrize("n,m", [(5, 900), (16, 16), (16, 2000), (32, 1100), (32, 10), (33, 500)])
def test_attend_one_sequence_of_few_heads(kind, n, m):
    # both sides of the rule that takes these as few rows: up to 128 rows of a KV head
    s = Setup(kind, 2, 4, 128, [(n, m)], block=16, seed=n)
    s.check(*s.run())
    s.check(*s.run(causal=False), causal=False)


def test_attend_long_prompt():
    s = Setup("bf16", 1, 4, 128, [(3000, 3000), (1, 5000), (700, 2100)], block=32, seed=5)
    s.check(*s.run())


@pytest.mark.parametrize("kind,n_seq,m", [("bf16", 1, 30000), ("q4", 1, 30000), ("bf16", 100, 300), ("q4", 70, 500),
                                          ("bf16", 3, 70000)])
def test_attend_many_keys_and_sequences(kind, n_seq, m):
    lens = [(1, max(1, (m * (i + 1)) // n_seq)) for i in range(n_seq)]
    s = Setup(kind, 2, 4, 128, lens, block=16, seed=n_seq)
    s.check(*s.run())


@pytest.mark.parametrize("kind", ["bf16", "q4", "f32"])
def test_attend_wrong_hints_cost_only_speed(kind):
    s = Setup(kind, 2, 4, 64, [(1, 500), (60, 333), (2, 2)], block=16, seed=3)
    for q, m in [(1, 1), (1, 500), (60, 1), (0, 0), (10 ** 6, 10 ** 6)]:
        out = torch.full_like(s.q, float("nan"))
        s.cache.attend(0, s.q, out, s.q_ptr, s.kv_len, max_q_len=q, max_kv_len=m)
        s.check(out, None)


@pytest.mark.parametrize("kind", ["bf16", "q4", "f32"])
def test_attend_scale_and_large_scores(kind):
    s = Setup(kind, 1, 4, 128, [(1, 400), (50, 160)], block=16, seed=8)
    s.check(*s.run(scale=0.01), scale=0.01)
    s.q.mul_(8)  # scores of some hundreds: the maximum has to be taken off
    s.check(*s.run())
    s.q.mul_(-1)
    s.check(*s.run())


@pytest.mark.parametrize("kind", ["bf16", "q4"])
@pytest.mark.parametrize("D", [64, 128])
def test_attend_few_rows_large_scores(kind, D):
    # nearly all weight on one key: channels whose code stands for zero are sums of the others'
    s = Setup(kind, 1, 4, D, [(1, 400), (2, 160), (1, 3000)], block=16, seed=8)
    for f in (8, -1):
        s.q.mul_(f)
        s.check(*s.run())


@pytest.mark.parametrize("kind", ["bf16", "q4"])
def test_attend_one_row_keeps_the_largest_weight_exact(kind):
    # values only behind key j, which has the largest score: the output is its weight
    # times them, rounded to bf16 (half a unit in the last of 8 places) from fp32 sums
    # (scores of at most 40 in 64 products: 2^-23 * 64 * 40; 2^-11 of it in all)
    m, D = 30000, 64
    s = Setup(kind, 2, 4, D, [(1, m)], block=16, seed=11)
    rows = s.rows_of[0]
    for j in (500, 10007, 15064, 20001, 29990):
        s.val[1] = 0
        if kind == "q4":
            s.cache.codes[0, 1] = 0x88
            c = torch.randint(1, 16, (2, D), generator=torch.Generator().manual_seed(j))
            scale = s.cache.scales[0, 1, :, rows[j]].float().cpu()  # [H, D / 32]
            s.val[1, rows[j]] = ((c - 8) * scale.repeat_interleave(32, -1)).to(s.val)
            s.cache.codes[0, 1, :, rows[j]] = torch.as_tensor(P.pack_codes(c.numpy().astype(np.uint8))).cuda()
        else:
            s.val[1, rows[j]] = torch.randn((2, D), generator=torch.Generator().manual_seed(j)).to(s.val)
        k = s.val[0, rows[j]].double()  # [H, D]
        f = torch.tensor([4.7, 5.0, 5.2, 5.5], device="cuda", dtype=torch.double)
        q = f[None, :, None] * 8 * (k / (k * k).sum(-1, keepdim=True))[:, None]
        s.q.copy_(q.reshape(1, 8, D).to(s.q.dtype))
        out, _ = s.run()
        o, _, _, _ = P.attend(s.q, s.val[0, rows], s.val[1, rows], True)
        half_unit = 2.0 ** (torch.floor(torch.log2(o.abs())) - 8)
        assert ((out.double() - o).abs() <= half_unit + 2.0 ** -11 * o.abs()).all(), j


@pytest.mark.parametrize("n", [1, 2, 70, 200])
def test_attend_strided_projections(n):
    # q, k, v as slices of one projection's output, outputs into a slice
    H, G, D = 2, 3, 64
    T = 2 * n + 1
    g = torch.Generator(device="cuda").manual_seed(n)
    qkv = torch.randn((T, (G + 2) * H + 1, D), generator=g, device="cuda").to(torch.bfloat16)
    q, k, v = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:H * G + 2 * H]
    big = torch.full((T, H * G, 2 * D), float("nan"), dtype=torch.bfloat16, device="cuda")
    cache = pipeline.KVCache.of_tensors(k, v, n_seq=2, row0=_i32([0, n]))
    cache.attend(0, q, big[..., :D], _i32([0, n, T]), _i32([n, n + 1]))
    torch.cuda.synchronize()
    for a, b in ((0, n), (n, T)):
        o, _, absv, size = P.attend(q[a:b], k[a:b], v[a:b], True)
        assert ((big[a:b, :, :D].double() - o).abs() <= P.bound(o, absv, size, torch.bfloat16)).all()
    assert torch.isnan(big[..., D:]).all()


@pytest.mark.parametrize("kind", ["bf16", "q4"])
@pytest.mark.parametrize("n", [1, 90])
def test_attend_same_bits_every_time(kind, n):
    s = Setup(kind, 2, 4, 128, [(n, 5000), (n, 777)], block=16, seed=1)
    a, e = s.run()
    for _ in range(3):
        b, f = s.run()
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(e, f)


@pytest.mark.parametrize("kind", ["bf16", "f32", "q4"])
@pytest.mark.parametrize("n", [1, 70])
def test_attend_bad_blocks_and_lengths_are_flagged(kind, n):
    s = Setup(kind, 1, 2, 64, [(n, 100)], block=16, seed=2)
    s.table[0, 3] = 10 ** 6
    out, _ = s.run()
    assert s.cache.status() & 0x08
    assert torch.isfinite(out.float()).all()
    s = Setup(kind, 1, 2, 64, [(n, 100)], block=16, seed=2)
    s.kv_len.fill_(10 ** 6)
    s.cache.attend(0, s.q, torch.empty_like(s.q), s.q_ptr, s.kv_len)
    assert s.cache.status() & 0x10


@pytest.mark.parametrize("n", [1, 70])
def test_attend_non_finite_rows(n):
    # an infinity or NaN that a query sees comes out as sums give it; a query of
    # another sequence, or of a later call, is not touched
    s = Setup("bf16", 1, 2, 64, [(n, 150), (n, 150)], block=16, seed=4)
    bad = s.rows_of[0][20]
    s.val[1, bad, 0, 3] = float("inf")
    out, _ = s.run()
    assert torch.isinf(out[n - 1, :, 3]).all() and torch.isfinite(out[n - 1, :, 4:].float()).all()
    o, _, absv, size = P.attend(s.q[n:], s.val[0, s.rows_of[1]], s.val[1, s.rows_of[1]], True)
    assert ((out[n:].double() - o).abs() <= P.bound(o, absv, size, s.dtype)).all()
    s.val[0, bad, 0, 3] = float("nan")
    out, _ = s.run()
    assert torch.isnan(out[n - 1].float()).all()
    assert ((out[n:].double() - o).abs() <= P.bound(o, absv, size, s.dtype)).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("kind,D,lens", [
    ("bf16", 64, [(4, 300), (2, 5)]), ("bf16", 128, [(3, 2000)]), ("q4", 64, [(4, 300)]), ("q4", 128, [(3, 2000)]),
    ("bf16", 64, [(70, 300), (33, 20)]), ("bf16", 128, [(200, 3000), (1, 64)]), ("bf16", 128, [(300, 300)]),
    ("q4", 64, [(200, 900)]), ("q4", 128, [(30, 4000)]), ("f32", 64, [(40, 100)]), ("bf16", 96, [(40, 100)])])
def test_attend_non_finite_rows_after_a_query(kind, D, lens, bad):
    # the last rows hold an infinity or NaN in a key's and a value's channel: queries
    # before them come out as if they were not there, the last ones with them
    s = Setup(kind, 2, 4, D, lens, block=16, seed=D)
    ends = np.cumsum([n for n, _ in lens])
    for rows in s.rows_of:
        at = rows[len(rows) - 1]
        if kind == "q4":
            s.cache.scales[0, :, 1, at, 0] = bad
        else:
            s.val[:, at, 1, 3] = bad
    out, _ = s.run(lse=False)
    first = 0
    for (n, m), rows, end in zip(s.lens, s.rows_of, ends):
        n1 = n - 1
        if n1 > 0:
            k, v = s.val[0, rows[:m - 1]], s.val[1, rows[:m - 1]]
            o, _, absv, size = P.attend(s.q[first:first + n1], k, v, True)
            assert ((out[first:first + n1].double() - o).abs() <= P.bound(o, absv, size, s.dtype)).all()
        assert torch.isfinite(out[end - 1, :4].float()).all() and torch.isnan(out[end - 1, 4:].float()).any()
        first = int(end)
    assert s.cache.status() == 0


@pytest.mark.parametrize("n", [1, 40])
def test_attend_rows_past_32_bit_offsets(n):
    # a pool of 2.4 million rows: the last rows lie past 2^31 elements and 2^32 bytes
    H, D, block = 8, 128, 16
    rows = 2_400_000
    kv = torch.zeros((1, 2, rows, H, D), dtype=torch.bfloat16, device="cuda")
    m = 333
    table = torch.arange(rows // block - 21, rows // block, dtype=torch.int32, device="cuda")[None].contiguous()
    g = torch.Generator(device="cuda").manual_seed(1)
    kv[0, :, rows - 21 * block:] = torch.randn((2, 21 * block, H, D), generator=g, device="cuda").to(torch.bfloat16)
    cache = pipeline.KVCache(kind="bf16", H=H, D=D, n_seq=1, kv=kv, block_table=table, block_size=block)
    q = torch.randn((n, 2 * H, D), generator=g, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    cache.attend(0, q, out, _i32([0, n]), _i32([m]), max_q_len=n, max_kv_len=m)
    k, v = kv[0, 0, rows - 21 * block:][:m], kv[0, 1, rows - 21 * block:][:m]
    o, _, absv, size = P.attend(q, k, v, True)
    assert ((out.double() - o).abs() <= P.bound(o, absv, size, torch.bfloat16)).all()
    assert cache.status() == 0


@pytest.mark.parametrize("kind", ["bf16", "q4"])
@pytest.mark.parametrize("n", [1, 50])
def test_attend_streams_and_graphs(kind, n):
    s = Setup(kind, 2, 4, 128, [(n, 900), (n, 60)], block=16, seed=6)
    a, _ = s.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.full_like(s.q, float("nan"))
    s.cache.attend(0, s.q, out, s.q_ptr, s.kv_len, max_q_len=n, max_kv_len=900, stream=side)
    side.synchronize()
    assert torch.equal(out, a)
    graph = torch.cuda.CUDAGraph()
    out2 = torch.full_like(s.q, float("nan"))
    with torch.cuda.graph(graph):
        s.cache.attend(0, s.q, out2, s.q_ptr, s.kv_len, max_q_len=n, max_kv_len=900)
    s.q.mul_(0.5)           # replays read the present queries and lengths
    s.kv_len.sub_(1)
    s.lens = [(n, m - 1) for _, m in s.lens]
    s.rows_of = [r[:-1] for r in s.rows_of]
    graph.replay()
    torch.cuda.synchronize()
    s.check(out2, None)


@pytest.mark.parametrize("kind", ["bf16", "f32", "q4"])
@pytest.mark.parametrize("n", [1, 40])
def test_attend_empty_cache(kind, n):
    c = pipeline.KVCache(kind=kind, H=2, D=64, n_seq=1, rows=0)
    q = torch.ones((n, 4, 64), dtype=TDT["f32" if kind == "f32" else "bf16"], device="cuda")
    out, lse = torch.full_like(q, 3.0), torch.zeros((n, 4), device="cuda")
    c.attend(0, q, out, _i32([0, n]), _i32([0]), lse=lse)
    assert (out == 0).all() and torch.isneginf(lse).all() and c.status() == 0


@pytest.mark.parametrize("kind", ["bf16", "q4"])
def test_attend_many_units_and_cuts(kind):
    # long enough that shares end inside units, at every kind of place
    for lens in ([(300, 4000), (1, 9000), (64, 2500)], [(40, 20000)], [(3, 3000)] * 7, [(2000, 2000), (0, 0), (129, 6000)]):
        s = Setup(kind, 2, 8, 64, lens, block=16, seed=len(lens))
        s.check(*s.run())
