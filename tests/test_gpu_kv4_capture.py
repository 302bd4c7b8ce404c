"""Calls of a 4-bit pool that are captured into a graph: a decode whose plan travels in the
parameters replays; whatever needs a staging slot, or changes the pool, is refused before it does."""
import pytest
import torch

from kv4_close import check, held

pytestmark = pytest.mark.gpu


def make(stlib, n, branches, seed=1):
    pool = stlib.Pool(n_layers=1, n_q_heads=8, n_kv_heads=2, head_dim=64, n_blocks=n // 16 + 3 * branches + 20,
                      max_seqs=branches + 4, max_decode_branches=branches, max_splits=16, kv_bits=4)
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn(n, 2, 64, generator=g).bfloat16() for _ in range(2))
    m = pool.seq_create()
    pool.append_kv([m], k[None, None].cuda(), v[None, None].cuda())
    return pool, [m] + pool.fork(m, branches - 1), held(k), held(v)


def rows(*shape, seed=3):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def test_calls_that_change_the_pool_are_refused(stlib):
    pool, br, k, v = make(stlib, 300, 3)
    q, kv = rows(1, 3, 8, 64), rows(1, 3, 2, 64, seed=4)
    for _ in range(10):  # every staging slot has been used
        f, = pool.fork(br[0], 1)
        pool.merge(f, q, kv, kv)
        pool.release(f)
    want = pool.decode_attn(br, q)
    pool.sync()
    before = pool.refcounts(), pool.free_list(), [pool.block_table(b) for b in br]
    o, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in (lambda: pool.append_kv(br, kv[:, :, None].contiguous(), kv[:, :, None].contiguous()),
                     lambda: pool.decode_step(br, kv, kv, q, o, lse), lambda: pool.merge(br[0], q, kv, kv),
                     lambda: pool.prefill_batch(br[:2], [1, 2], q, kv, kv)):
            with pytest.raises(stlib.STError) as e:
                call()
            assert e.value.status == stlib.ST_ERR_STATE
        pool.decode_attn(br, q, o, lse)
    assert before == (pool.refcounts(), pool.free_list(), [pool.block_table(b) for b in br])
    q2 = rows(1, 3, 8, 64, seed=5)
    q.copy_(q2)
    graph.replay()
    torch.cuda.synchronize()
    check(o[0], lse[0], q2[0], [(k, v)] * 3)
    pool.append_kv(br, kv[:, :, None].contiguous(), kv[:, :, None].contiguous())
    pool.merge(br[0], q, kv, kv)
    pool.sync()


def test_tables_that_have_changed_are_not_captured(stlib):
    """A fork's table goes out with the next call: outside of a graph."""
    pool, br, k, v = make(stlib, 100, 2)
    q = rows(1, 2, 8, 64)
    o, lse = torch.empty(1, 2, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 2, 8, device="cuda")
    back = torch.empty(1, 100, 2, 64, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o.zero_()
        for call in (lambda: pool.decode_attn(br, q, o, lse), lambda: pool.read_kv(br[1], 0, 100, back, back.clone())):
            with pytest.raises(stlib.STError) as e:
                call()
            assert e.value.status == stlib.ST_ERR_STATE
    pool.decode_attn(br, q, o, lse)
    pool.sync()
    check(o[0], lse[0], q[0], [(k, v)] * 2)
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        pool.decode_attn(br, q, o, lse)
        pool.read_kv(br[1], 0, 100, back, torch.empty_like(back))


def test_a_plan_too_large_for_the_parameters_is_not_captured(stlib):
    pool, br, k, v = make(stlib, 400, 100)
    q = rows(1, 100, 8, 64)
    for _ in range(12):  # every staging slot has been used
        o, lse = pool.decode_attn(br, q)
    pool.sync()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        torch.empty(1, device="cuda").zero_()
        with pytest.raises(stlib.STError) as e:
            pool.decode_attn(br, q, o, lse)
        assert e.value.status == stlib.ST_ERR_STATE
    for _ in range(12):  # and goes on
        o, lse = pool.decode_attn(br, q)
    pool.sync()
    check(o[0][:3], lse[0][:3], q[0][:3], [(k, v)] * 3)
