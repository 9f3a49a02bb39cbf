"""What the calls on a cache refuse on the host, before anything touches a GPU."""

import ctypes

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2609_32259_gb300 import build, binding

    build.build()
    binding.lib()
    return binding


def _cache(B, **over):
    kw = dict(kind=0, H=2, D=64, n_seq=1, rows=100, d_k=4096, d_v=8192)
    kw.update(over)
    return B.CacheDesc(**kw)


CACHE_REFUSALS = [
    (dict(kind=3), 1), (dict(H=0), 1), (dict(D=48), 2), (dict(kind=2, D=32, d_k_scale=16, d_v_scale=16), 2),
    (dict(D=512), 2), (dict(n_seq=0), 1), (dict(n_seq=1025), 1), (dict(rows=-1), 1), (dict(rows=1 << 31), 1),
    (dict(d_k=None), 1), (dict(d_v=None), 1), (dict(d_k=4100), 1), (dict(kind=2), 1),
    (dict(kind=2, d_k_scale=16, d_v_scale=16, row_stride=128), 1), (dict(row_stride=129), 1),
    (dict(head_stride=-64), 1), (dict(d_block_table=64, block_size=0, max_blocks_per_seq=4), 1),
    (dict(d_block_table=64, block_size=16, max_blocks_per_seq=4), 1),  # 16 does not divide 100 rows
    (dict(d_block_table=64, block_size=10, max_blocks_per_seq=0), 1), (dict(n_seq=2), 1),
]


@pytest.mark.parametrize("over,status", CACHE_REFUSALS)
def test_caches(B, over, status):
    c = _cache(B, **over)
    a = B.AppendDesc(dtype=0, n_tok=0)
    r = B.ReadDesc(dtype=0, n_tok=0)
    n = ctypes.c_size_t(0)
    L = B.lib()
    assert L.hf_cache_append(ctypes.byref(c), ctypes.byref(a), None) == status
    assert L.hf_cache_read(ctypes.byref(c), ctypes.byref(r), None) == status
    assert L.hf_attend_workspace_size(ctypes.byref(c), ctypes.byref(n)) == status
    assert L.hf_attend(ctypes.byref(c), ctypes.byref(B.AttendDesc(dtype=0, H_q=2)), 256, 1 << 40, None) == status
    assert L.hf_last_error()


def test_null_descriptors(B):
    L, c = B.lib(), _cache(B)
    assert L.hf_cache_append(None, None, None) == 1
    assert L.hf_cache_append(ctypes.byref(c), None, None) == 1
    assert L.hf_cache_read(ctypes.byref(c), None, None) == 1
    assert L.hf_attend(ctypes.byref(c), None, None, 0, None) == 1
    assert L.hf_attend_workspace_size(ctypes.byref(c), None) == 1


@pytest.mark.parametrize("over", [
    dict(dtype=2), dict(dtype=1), dict(n_tok=-1), dict(d_tok_ptr=None), dict(d_start=None), dict(d_k=None),
    dict(d_v=None), dict(d_k=4104), dict(k_row_stride=100), dict(v_head_stride=4), dict(d_q=64, H_q=0, d_q_out=64),
    dict(d_q=64, H_q=4), dict(d_q=72, H_q=4, d_q_out=64), dict(d_rope=64, rope_len=0), dict(d_rope=68, rope_len=5),
    dict(d_k_norm=64, eps=-1.0), dict(d_k_norm=64, eps=float("nan")), dict(d_q=64, d_q_out=64, H_q=4, q_row_stride=3),
    dict(d_q=64, d_q_out=128, H_q=4, q_out_head_stride=-64), dict(d_q=64, d_q_out=64, H_q=4, q_out_row_stride=512),
])
def test_appends(B, over):
    kw = dict(dtype=0, n_tok=5, d_tok_ptr=64, d_start=64, d_k=4096, d_v=4096)
    kw.update(over)
    c = _cache(B)
    assert B.lib().hf_cache_append(ctypes.byref(c), ctypes.byref(B.AppendDesc(**kw)), None) == 1


@pytest.mark.parametrize("over", [dict(dtype=1), dict(n_tok=-1), dict(d_tok_ptr=None), dict(d_k=None), dict(d_v=24),
                                  dict(k_row_stride=3)])
def test_reads(B, over):
    kw = dict(dtype=0, n_tok=5, d_tok_ptr=64, d_start=64, d_k=4096, d_v=4096)
    kw.update(over)
    c = _cache(B)
    assert B.lib().hf_cache_read(ctypes.byref(c), ctypes.byref(B.ReadDesc(**kw)), None) == 1


@pytest.mark.parametrize("over,status", [
    (dict(dtype=2), 1), (dict(dtype=1), 1), (dict(H_q=0), 1), (dict(H_q=3), 1), (dict(H_q=2 * 257), 1),
    (dict(n_tok=-1), 1), (dict(max_q_len=-1), 1), (dict(max_kv_len=-1), 1), (dict(causal=2), 1),
    (dict(scale=-1.0), 1), (dict(scale=float("inf")), 1), (dict(d_q_ptr=None), 1), (dict(d_kv_len=None), 1),
    (dict(d_q=None), 1), (dict(d_out=None), 1), (dict(d_q=8), 1), (dict(d_out=8), 1), (dict(q_row_stride=5), 1),
    (dict(out_head_stride=-8), 1), (dict(n_tok=1 << 30), 1),
    (dict(ws=None), 6), (dict(ws=128), 6), (dict(ws_bytes=1000), 6),
])
def test_attends(B, over, status):
    kw = dict(dtype=0, H_q=4, n_tok=5, d_q_ptr=64, d_kv_len=64, max_q_len=5, max_kv_len=50, causal=1, d_q=4096,
              d_out=8192, ws=256, ws_bytes=1 << 40)
    kw.update(over)
    ws, nb = kw.pop("ws"), kw.pop("ws_bytes")
    c = _cache(B)
    assert B.lib().hf_attend(ctypes.byref(c), ctypes.byref(B.AttendDesc(**kw)), ws, nb, None) == status


@pytest.mark.parametrize("args", [(63, 1e4, 0, 5, 64), (0, 1e4, 0, 5, 64), (512, 1e4, 0, 5, 64), (64, 0.0, 0, 5, 64),
                                  (64, 1e4, -1, 5, 64), (64, 1e4, 1 << 24, 1, 64), (64, 1e4, 0, -1, 64),
                                  (64, 1e4, 0, 5, None), (64, 1e4, 0, 5, 72)])
def test_rope_tables(B, args):
    D, theta, pos0, n, p = args
    assert B.lib().hf_rope_table(D, theta, None, pos0, n, p, None) == 1


def test_nothing_to_do_is_no_error(B):
    L, c = B.lib(), _cache(B)
    assert L.hf_cache_append(ctypes.byref(c), ctypes.byref(B.AppendDesc(dtype=0)), None) == 0
    assert L.hf_cache_read(ctypes.byref(c), ctypes.byref(B.ReadDesc(dtype=0)), None) == 0
    assert L.hf_attend(ctypes.byref(c), ctypes.byref(B.AttendDesc(dtype=0, H_q=2)), 256, 1 << 40, None) == 0
    assert L.hf_rope_table(64, 1e4, None, 0, 0, None, None) == 0


def test_tensors_of_the_wrong_kind():
    import torch

    from paper_2609_32259_gb300.pipeline import KVCache

    with pytest.raises(ValueError):
        KVCache(kind="bf16", H=2, D=64, n_seq=1, kv=torch.zeros((1, 2, 10, 2, 64)))  # fp32
    with pytest.raises(ValueError):
        KVCache(kind="q4", H=2, D=64, n_seq=1, codes=torch.zeros((1, 2, 2, 10, 32), dtype=torch.uint8),
                scales=torch.zeros((1, 2, 2, 10, 2)))
    with pytest.raises(KeyError):
        KVCache(kind="int8", H=2, D=64, n_seq=1, rows=4, device="cpu")
    c = KVCache(kind="bf16", H=2, D=64, n_seq=1, rows=16, device="cpu")
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        c.append(0, k, k.float(), i, i[:1])
    with pytest.raises(ValueError):
        c.append(0, k, k.transpose(0, 1), i, i[:1])
    with pytest.raises(ValueError):
        c.append(0, k[:, :1].expand(3, 2, 64), k, i, i[:1])  # one head's row for both
    with pytest.raises(ValueError):
        c.append(0, k.half(), k.half(), i, i[:1])
    with pytest.raises(ValueError):
        c.append(0, k, k, i.long(), i[:1])
    with pytest.raises(ValueError):
        c.append(0, k, k, i, i[:1], q=k)
    with pytest.raises(ValueError):
        c.append(0, k, k, i, i[:1], rope=torch.zeros((4, 64)))
    with pytest.raises(ValueError):
        c.attend(0, k, k.float(), i, i[:1])
    with pytest.raises(ValueError):
        c.attend(0, k, k, i, i[:1], lse=torch.zeros(3))
    with pytest.raises(ValueError):
        KVCache.of_tensors(k, k.float())
