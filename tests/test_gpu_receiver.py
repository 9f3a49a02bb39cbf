"""A transfer, a question and decoding steps behind it, through ReceiverSteps,
against the 64-bit form over the transferred rows and the appended ones."""

import numpy as np
import pytest
import torch

import cache_plain as P
from oracle import heterofold_oracle as O
from paper_2609_32259_gb300 import pipeline, receiver
from paper_2609_32259_gb300 import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as g

    g.build()


@pytest.mark.parametrize("kind", ["bf16", "q4"])
def test_question_and_steps_behind_a_transfer(kind):
    dev = torch.device("cuda")
    direction = W.llama_to_qwen25(200).with_(L_s=5, L_r=3, name="receiver_steps")
    new = [23, 1, 1]
    w, T, job = receiver._paged_job(direction, sum(new), dev)
    job.step()
    torch.cuda.synchronize()
    assert job.align_status() == 0 and job.device_status() == 0
    cache = pipeline.KVCache.of_job(job)
    H, D, G = w.H_r, w.D_r, 7
    rows = (torch.as_tensor(job.paged.block_table[0]).cuda().long()[:, None] * w.block_size
            + torch.arange(w.block_size, device=dev)).reshape(-1)[:T]
    # what the cache holds of the context (the transfer itself is compared elsewhere)
    kv = job.receiver.view(w.L_r, 2, -1, H, D)[:, :, rows].double()
    if kind == "q4":
        cache = receiver.packed_in_4_bits(cache, [T])
        kv = torch.as_tensor(P.held_in_4_bits(kv.float().cpu().numpy())[0]).cuda()
    rope = pipeline.rope_table(T + sum(new), D, theta=w.theta_r)
    rec = receiver.ReceiverSteps(cache, [T], rope)
    g = torch.Generator(device="cuda").manual_seed(2)
    for n in new:
        rec.begin([n])
        for l in range(w.L_r):
            qkv = torch.randn((n, H * (G + 2), D), generator=g, device="cuda").to(torch.bfloat16)
            q, k, v = qkv[:, :H * G], qkv[:, H * G:H * G + H], qkv[:, H * G + H:]
            out = rec.layer(l, q, k, v)
            pos = np.arange(int(rec.lens[0]), int(rec.lens[0]) + n)
            f = O.rope_inv_freq(w.theta_r, D)
            qr = torch.as_tensor(P.rotated(q.double().cpu().numpy(), pos, f)).cuda().to(torch.bfloat16).double()
            # the rows as the cache holds them: their rounding is tested with append
            ptr, start = rec.tok_ptr, rec.start
            ko, vo = torch.empty((n, H, D), dtype=torch.bfloat16, device="cuda"), torch.empty(
                (n, H, D), dtype=torch.bfloat16, device="cuda")
            cache.read(l, ko, vo, ptr, start)
            if l == 0:
                new_k = torch.empty((w.L_r, n, H, D), dtype=torch.float64, device="cuda")
                new_v = torch.empty_like(new_k)
            new_k[l], new_v[l] = ko.double(), vo.double()
            keys = torch.cat([kv[l, 0], new_k[l]])
            vals = torch.cat([kv[l, 1], new_v[l]])
            o, _, absv, size = P.attend(qr, keys, vals, True)
            # a rotated query may round to the other neighbour: 2^-8 of its scores
            tol = P.bound(o, absv, size, torch.bfloat16) + 2.0 ** -8 * size[..., None] * absv
            assert ((out.double() - o).abs() <= tol).all()
            assert (ko.double() - torch.as_tensor(P.rotated(k.double().cpu().numpy(), pos, f)).cuda()).abs().max() <= (
                0.02 if kind == "bf16" else 0.6)
        kv = torch.cat([kv, torch.stack([new_k, new_v], 1)], 2)
        rec.end()
    assert cache.status() == 0 and rec.lens.tolist() == [T + sum(new)]


def test_steps_are_checked():
    cache = pipeline.KVCache(kind="bf16", H=1, D=64, n_seq=2, rows=64, row0=torch.tensor([0, 32], dtype=torch.int32,
                                                                                         device="cuda"))
    rope = pipeline.rope_table(32, 64, theta=1e4)
    with pytest.raises(ValueError):
        receiver.ReceiverSteps(cache, [1], rope)
    rec = receiver.ReceiverSteps(cache, [3, 30], rope)
    with pytest.raises(ValueError):
        rec.begin([1, 3])  # past the rotation table
    with pytest.raises(ValueError):
        rec.begin([-1, 1])
    x = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        rec.layer(0, x, x, x)
