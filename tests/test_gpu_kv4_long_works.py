"""A prefill whose single works take longer than a device-side wait's limit of 2 s: no wait may
span a whole work.  268 million keys of one head of 64, 18 GB of pages, three works a block."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_works_of_seconds(stlib):
    n, T, G, D, piece = 1 << 28, 815, 48, 64, 1 << 23
    pool = stlib.Pool(n_layers=1, n_q_heads=G, n_kv_heads=1, head_dim=D, n_blocks=(n + T) // 16 + 2, max_seqs=2,
                      max_decode_branches=1, max_splits=2, kv_bits=4)
    s = pool.seq_create()
    k = torch.zeros(1, 1, piece, 1, D, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, 1.75)
    for _ in range(n // piece):
        pool.append_kv([s], k, v)
    q = torch.ones(1, T, G, D, dtype=torch.bfloat16, device="cuda")
    k, v = k[:, 0, :T].contiguous(), v[:, 0, :T].contiguous()
    pool.sync()
    pool.profile_read()
    o, lse = pool.merge(s, q, k, v)
    pool.sync()
    got = pool.profile_read()["merge_prefill"]
    # 306 works on 152 SMs or so, whole, with three of them in some blocks
    assert got["kernels"] == 1
    # Equal keys, values held as they are (7 times a quarter): the log-sum-exp sums 2^21 equal weights a thread,
    # exactly.  O is summed 2^28 / 16 times in the tensor core, each step cut off at 2^-23 of the sum, twice
    # the sum in all: no more can be asked of it at this length than that it is no larger than the values.
    assert ((o > 0) & (o <= 1.75)).all()
    want = torch.log(torch.arange(n + 1, n + T + 1, dtype=torch.float64)).view(1, T, 1)
    assert ((lse.double().cpu() - want).abs() <= 2.0 ** -18 * math.log(n)).all()
