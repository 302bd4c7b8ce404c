"""Rows of a tile are independent: a query that is far larger or smaller than those beside it
leaves their results what they would be alone, against the float64 oracle over the values held
(tolerances: kv4_close.py, each row by its own queries and keys)."""
import pytest
import torch

from kv4_close import check, held

pytestmark = pytest.mark.gpu


def drawn(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def one_sequence(stlib, n, Hq, Hkv, D, seed, **kw):
    """A pool with one sequence of n rows, and its context as held."""
    pool = stlib.Pool(n_layers=1, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, n_blocks=n // 16 + 120, max_seqs=40,
                      kv_bits=4, **kw)
    k, v = drawn(n, Hkv, D, seed=seed).bfloat16(), drawn(n, Hkv, D, seed=seed + 1).bfloat16()
    s = pool.seq_create()
    pool.append_kv([s], k[None, None].cuda(), v[None, None].cuda())
    return pool, s, held(k), held(v)


# from 2^-120 to 2^96 of an ordinary row, and rows that are all zeros
def sizes(n, seed):
    e = torch.randint(-30, 25, (n,), generator=torch.Generator().manual_seed(seed)).double() * 4
    e[::3] = 0  # ordinary ones among them
    by = 2.0 ** e
    by[5::11] = 0
    return by


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ratio", [2.0 ** 24, 2.0 ** 31, 2.0 ** 36, 2.0 ** 40, 1e20, 1e30])
def test_a_large_finite_query_leaves_its_neighbours_alone(stlib, D, ratio):
    pool, s, k, v = one_sequence(stlib, 700, 8, 1, D, 3)
    q = drawn(1, 1, 8, D, seed=9)
    q[0, 0, 2] *= ratio
    q = q.bfloat16()
    o, lse = pool.decode_attn([s], q.cuda())
    pool.sync()
    rest = [0, 1, 3, 4, 5, 6, 7]
    check(o[0][:, rest], lse[0][:, rest], q[0][:, rest], [(k, v)])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("branches", [5, 8, 12, 20])
def test_decode_of_unlike_rows(stlib, D, branches):
    """Narrow and wide works, and two subgroups; sizes drawn row by row, ordinary ones checked."""
    pool, s, k, v = one_sequence(stlib, 1200, 8, 1, D, 4, max_decode_branches=20)
    br = [s] + pool.fork(s, branches - 1)
    by = sizes(branches * 8, branches).view(branches, 8, 1)
    q = (drawn(1, branches, 8, D, seed=11) * by).bfloat16()
    o, lse = pool.decode_attn(br, q.cuda())
    pool.sync()
    small = by.view(branches, 8) <= 1
    for b in range(branches):
        h = torch.nonzero(small[b]).flatten().tolist()
        check(o[0, b:b + 1, h], lse[0, b:b + 1, h], q[0, b:b + 1, h], [(k, v)], f"branch {b}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 8, 9, 40, 133])
def test_prefill_of_unlike_rows(stlib, D, T):
    pool, s, k, v = one_sequence(stlib, 900, 8, 1, D, 5)
    by = sizes(T * 8, T).view(T, 8, 1)
    q = (drawn(1, T, 8, D, seed=12) * by).bfloat16()
    nk, nv = drawn(T, 1, D, seed=13).bfloat16(), drawn(T, 1, D, seed=14).bfloat16()
    o, lse = pool.merge(s, q.cuda(), nk[None].cuda(), nv[None].cuda())
    pool.sync()
    k, v = torch.cat([k, held(nk)]), torch.cat([v, held(nv)])
    small = by.view(T, 8) <= 1
    for t in range(0, T, max(1, T // 12)):
        h = torch.nonzero(small[t]).flatten().tolist()
        if h:
            check(o[0, t:t + 1, h], lse[0, t:t + 1, h], q[0, t:t + 1, h], [(k[:900 + t + 1], v[:900 + t + 1])], f"row {t}")


def test_a_row_is_the_same_whatever_is_beside_it(stlib):
    """Bitwise: a row's scale is its own."""
    pool, s, k, v = one_sequence(stlib, 2000, 8, 2, 128, 6)
    q = drawn(1, 1, 8, 128, seed=15)
    a, la = pool.decode_attn([s], q.bfloat16().cuda())
    q[0, 0, 1] *= 2.0 ** 12
    q[0, 0, 6] *= 2.0 ** -20
    b, lb = pool.decode_attn([s], q.bfloat16().cuda())
    pool.sync()
    rest = [0, 2, 3, 4, 5, 7]
    assert torch.equal(a[0, 0, rest], b[0, 0, rest]) and torch.equal(la[0, 0, rest], lb[0, 0, rest])
