"""hf_cache_append, hf_cache_read and hf_rope_table against 64-bit forms: every
cache kind and width, norms, rotation, layouts, the rows around the written ones,
special values of the 4-bit format, refused rows."""

import numpy as np
import pytest
import torch

import cache_plain as P
from oracle import heterofold_oracle as O
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


def _make(kind, H, D, lens, block, seed=0):
    """A cache of marked rows for sequences of (tokens, rows before them)."""
    n = len(lens)
    total = [a + b for a, b in lens]
    g = torch.Generator(device="cuda").manual_seed(seed)
    if block:
        need = [-(-t // block) for t in total]
        nb = sum(need) + 2
        perm = torch.randperm(nb, generator=g, device="cuda").to(torch.int32)
        table = torch.full((n, max(max(need), 1)), 10 ** 9, dtype=torch.int32, device="cuda")
        at = 0
        for i, c in enumerate(need):
            table[i, :c] = perm[at:at + c]
            at += c
        rows, row0 = nb * block, None
        of = [(table[i].long()[:, None] * block + torch.arange(block, device="cuda")).reshape(-1)[:t]
              for i, t in enumerate(total)]
    else:
        st = np.cumsum([0] + [t + 3 for t in total])
        rows, row0, table = int(st[-1]), _i32(st[:-1]), None
        of = [torch.arange(int(st[i]), int(st[i]) + t, device="cuda") for i, t in enumerate(total)]
    cache = pipeline.KVCache(kind=kind, H=H, D=D, n_seq=n, rows=rows, layers=2, block_table=table, block_size=block,
                             row0=row0)
    if kind == "q4":
        cache.codes.fill_(0x5a)
        cache.scales.fill_(0.375)
    else:
        cache.kv.fill_(-7.0)
    new = torch.cat([r[b:] for r, (a, b) in zip(of, lens)])
    ptr = _i32(np.concatenate([[0], np.cumsum([a for a, _ in lens])]))
    start = _i32([b for _, b in lens])
    pos = np.concatenate([np.arange(b, a + b) for a, b in lens])
    return cache, new, ptr, start, pos, g


LENS = [(1, 0), (0, 4), (37, 5), (16, 16), (5, 300)]


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("kind,H,Hq,D,block", [
    ("bf16", 8, 32, 128, 16), ("bf16", 1, 7, 64, 0), ("bf16", 3, 3, 32, 24), ("bf16", 2, 4, 96, 8),
    ("bf16", 1, 2, 256, 64), ("f32", 4, 8, 32, 16), ("f32", 2, 6, 128, 0), ("f32", 1, 1, 256, 1),
    ("f32", 5, 5, 64, 16), ("f32", 1, 2, 96, 0),
])
def test_append_and_read(kind, H, Hq, D, block, norm):
    cache, new, ptr, start, pos, g = _make(kind, H, D, LENS, block, seed=H * D)
    T, dt = len(pos), TDT[kind]
    k, v = (torch.randn((T, H, D), generator=g, device="cuda").to(dt) for _ in range(2))
    q = torch.randn((T, Hq, D), generator=g, device="cuda").to(dt)
    kn, qn = (torch.randn(D, generator=g, device="cuda") if norm else None for _ in range(2))
    rope = pipeline.rope_table(400, D, theta=1e4)
    before = cache.kv.clone()
    q_out = torch.full_like(q, float("nan"))
    cache.append(1, k, v, ptr, start, rope=rope, q=q, q_out=q_out, k_norm=kn, q_norm=qn)
    assert cache.status() == 0
    f = O.rope_inv_freq(1e4, D)
    # one rounding to the type; in fp32 sums of D squares, two products and their
    # sum, and angles to 1e-6 rad with sines to 4e-7
    rel, ab = (2.0 ** -8, 4e-6) if kind == "bf16" else (2.0 ** -20, 4e-6)

    def close(got, ref):
        size = np.abs(ref).max(-1, keepdims=True)
        assert (np.abs(got.double().cpu().numpy() - ref) <= rel * np.abs(ref) + ab * size + 1e-30).all()

    tn = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    close(cache.kv[1, 0, new], P.rotated(tn(k), pos, f, tn(kn)))
    close(q_out, P.rotated(tn(q), pos, f, tn(qn)))
    assert torch.equal(cache.kv[1, 1, new], v)
    cache.kv[1, :, new] = before[1, :, new]
    assert torch.equal(cache.kv, before)  # no other row, no other layer
    # reading back, into strided destinations
    cache.append(0, k, v, ptr, start)
    ko = torch.zeros((T, 2 * H, D), dtype=dt, device="cuda")
    cache.read(0, ko[:, :H], ko[:, H:], ptr, start)
    assert torch.equal(ko[:, :H], k) and torch.equal(ko[:, H:], v)
    # queries in place
    q2 = q.clone()
    cache.append(1, k, v, ptr, start, rope=rope, q=q2, q_out=q2, k_norm=kn, q_norm=qn)
    assert torch.equal(q2, q_out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,D,block", [(8, 128, 16), (1, 64, 0), (3, 64, 8), (5, 128, 24), (2, 256, 16), (9, 128, 1)])
def test_append_4_bits(H, D, block, dtype):
    cache, new, ptr, start, pos, g = _make("q4", H, D, LENS, block, seed=D + H)
    T, dt = len(pos), TDT[dtype]
    k, v = ((torch.randn((T, H, D), generator=g, device="cuda")
             * 10 ** (torch.rand((H, D), generator=g, device="cuda") * 2 - 1)).to(dt) for _ in range(2))
    q = torch.randn((T, 3 * H, D), generator=g, device="cuda").to(dt)
    v[0, 0, :32] = 0                      # a group of zeros
    v[1, 0, :32] = 1e-37                  # below what a scale holds
    v[2, 0, 32:64] = torch.linspace(-3.5, 3.5, 32, device="cuda").to(dt)  # ties of rint(y / 0.5)
    rope = pipeline.rope_table(400, D, theta=1e4)
    codes0, scales0 = cache.codes.clone(), cache.scales.clone()
    q_out = torch.empty_like(q)
    cache.append(1, k, v, ptr, start, rope=rope, q=q, q_out=q_out)
    assert cache.status() == 0
    # the rotation as defined: every product and sum rounded to fp32
    t = rope.cpu().numpy()[pos][:, None]
    c, s = t[..., 0], t[..., 1]
    kf = k.float().cpu().numpy()
    a, b = kf[..., :D // 2], kf[..., D // 2:]
    kr = np.concatenate([a * c - b * s, b * c + a * s], -1)
    assert kr.dtype == np.float32
    for which, x in ((0, kr), (1, v.float().cpu().numpy())):
        val, code, sc = P.held_in_4_bits(x)
        got = cache.codes[1, which].permute(1, 0, 2)[new].cpu().numpy()
        assert np.array_equal(got, P.pack_codes(code))
        assert np.array_equal(cache.scales[1, which].permute(1, 0, 2)[new].float().cpu().numpy(), sc)
        # what is read is what the codes stand for, exactly, in either type
        for odt in ("bf16", "f32"):
            ko, vo = (torch.empty((T, H, D), dtype=TDT[odt], device="cuda") for _ in range(2))
            cache.read(1, ko, vo, ptr, start)
            assert np.array_equal((ko, vo)[which].double().cpu().numpy(), val)
        # half a step, and what the scale's own rounding (2^-5) leaves past code 7
        step = np.repeat(sc, 32, -1).reshape(x.shape)
        assert (np.abs(val - x) <= 0.5 * step * (1 + 2.0 ** -4) + 8e-31).all()
    cache.codes[1][:, :, new], cache.scales[1][:, :, new] = codes0[1][:, :, new], scales0[1][:, :, new]
    assert torch.equal(cache.codes, codes0) and torch.equal(cache.scales, scales0)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_4_bit_groups_with_non_finite_values(bad):
    cache, new, ptr, start, pos, g = _make("q4", 2, 64, [(3, 0)], 0)
    k = torch.randn((3, 2, 64), generator=g, device="cuda").to(torch.bfloat16)
    v = k.clone()
    v[1, 1, 40] = bad
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    cache.append(0, k, v, ptr, start)
    cache.read(0, ko, vo, ptr, start)
    nan = torch.isnan(vo)
    assert nan[1, 1, 32:].all() and int(nan.sum()) == 32 and torch.isfinite(ko.float()).all()


def test_pack_a_transferred_cache():
    # a contiguous bf16 cache, already rotated, into 4 bits and back, all at once
    rows, H, D = 1000, 4, 128
    kv = torch.randn((1, 2, rows, H, D), device="cuda").to(torch.bfloat16)
    cache = pipeline.KVCache(kind="q4", H=H, D=D, n_seq=1, rows=rows)
    ptr, start = _i32([0, rows]), _i32([0])
    cache.append(0, kv[0, 0], kv[0, 1], ptr, start)
    out = torch.empty_like(kv)
    cache.read(0, out[0, 0], out[0, 1], ptr, start)
    val, _, _ = P.held_in_4_bits(kv.float().cpu().numpy())
    assert np.array_equal(out.double().cpu().numpy(), val)


def test_positions_behind_an_offset():
    cache, new, ptr, start, pos, g = _make("f32", 2, 64, [(4, 3), (2, 0)], 16)
    k = torch.randn((6, 2, 64), generator=g, device="cuda")
    rope = pipeline.rope_table(2000, 64, theta=1e4)
    cache.append(0, k, k, ptr, start, rope=rope, pos0=_i32([100, 1900]))
    p = np.concatenate([np.arange(103, 107), np.arange(1900, 1902)])
    ref = P.rotated(k.double().cpu().numpy(), p, O.rope_inv_freq(1e4, 64))
    assert np.abs(cache.kv[0, 0, new].double().cpu().numpy() - ref).max() <= 2e-5


@pytest.mark.parametrize("what,bit", [("block", 0x08), ("rows", 0x10), ("position", 0x10), ("pointers", 0x01)])
@pytest.mark.parametrize("kind", ["bf16", "q4"])
def test_rows_that_cannot_be_written(kind, what, bit):
    cache, new, ptr, start, pos, g = _make(kind, 2, 64, [(40, 0)], 16)
    k = torch.randn((40, 2, 64), generator=g, device="cuda").to(torch.bfloat16)
    rope = pipeline.rope_table(40 if what != "position" else 30, 64, theta=1e4)
    cache.append(0, k, k, ptr, start, rope=rope)
    store = cache.codes if kind == "q4" else cache.kv
    if what == "position":
        assert cache.status() == bit
        return
    before = store.clone()
    if what == "block":
        cache.block_table.fill_(-1)
    elif what == "rows":
        start.fill_(48)
        rope = pipeline.rope_table(1000, 64, theta=1e4)
    else:
        ptr[0] = 50
    cache.append(0, k + 1, k + 1, ptr, start, rope=rope)
    assert cache.status() == bit
    assert torch.equal(store, before)
    ko = torch.full_like(k, 5.0)
    if what != "pointers":
        cache.read(0, ko, ko.clone(), ptr, start)
        assert (ko == 0).all()


def test_rope_table_angles():
    for theta, D, pos0, n in ((5e5, 128, 0, 5000), (1e4, 64, 130000, 300), (1e8, 256, 16000000, 50)):
        t = pipeline.rope_table(n, D, theta=theta, pos0=pos0).double().cpu().numpy()
        ang = np.arange(pos0, pos0 + n)[:, None] * O.rope_inv_freq(theta, D).astype(np.float64)[None]
        assert np.abs(t[..., 0] - np.cos(ang)).max() <= 2e-6 and np.abs(t[..., 1] - np.sin(ang)).max() <= 2e-6
    f = np.linspace(0.1, 1.0, 16, dtype=np.float32)
    t = pipeline.rope_table(7, 32, inv_freq=f).double().cpu().numpy()
    assert np.abs(t[..., 1] - np.sin(np.arange(7)[:, None] * f.astype(np.float64))).max() <= 2e-6


def test_many_sequences():
    lens = [(i % 3, i % 7) for i in range(200)]
    cache, new, ptr, start, pos, g = _make("bf16", 2, 64, lens, 8)
    k = torch.randn((len(pos), 2, 64), generator=g, device="cuda").to(torch.bfloat16)
    cache.append(0, k, -k, ptr, start)
    assert cache.status() == 0
    assert torch.equal(cache.kv[0, 0, new], k) and torch.equal(cache.kv[0, 1, new], -k)
