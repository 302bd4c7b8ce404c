"""Queries and keys so large that the scores are beyond what fp32 tells apart: O stays a mean of the
values, the log-sum-exp within its tolerance (kv4_close.py), and where one key is ahead of all
others by more than the scores are off, O is that key's value."""
import numpy as np
import pytest
import torch

from kv4_close import attend, beyond, held

pytestmark = pytest.mark.gpu


def drawn(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def check_huge(o, lse, q, k, v, what=""):
    """o, lse [Hq, D], [Hq] of q [Hq, D] over k, v [n, Hkv, D]."""
    want = attend(q, k, v)
    over_o, over_lse = beyond(o.double().cpu().numpy(), lse.double().cpu().numpy(), want)
    e = want[2]
    g = q.shape[0] // k.shape[1]
    lo, hi = v.double().numpy().min(0).repeat(g, 0), v.double().numpy().max(0).repeat(g, 0)
    got, wide = o.double().cpu().numpy(), 2.0 ** -7 * np.abs(v.double().numpy()).max()
    assert ((got >= lo - wide) & (got <= hi + wide)).all(), f"{what}: not a mean of the values"
    assert (over_o <= 0).all() and (over_lse <= 0).all(), f"{what}: {over_o.max()} {over_lse.max()}"
    x = np.einsum("hd,nhd->hn", q.double().numpy(), k.double().numpy().repeat(g, 1)) / np.sqrt(q.shape[1])
    s = np.sort(x, 1)
    for h in range(q.shape[0]):  # exp(-30) of the weight for the rest: below a tenth of bf16's half step
        if x.shape[1] == 1 or s[h, -1] - s[h, -2] > 2 * e[h] + 30:
            best = v[int(x[h].argmax()), h // g].double().numpy()
            assert (np.abs(got[h] - best) <= 2.0 ** -8 * np.abs(best) + 2.0 ** -10 * np.abs(best).max()).all(), (what, h)


SIZES = [1e4, 1e6, 3e7, 1e8, 1e9, 1e12, 1e20, 1e30, 3e33]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("D,Hq,n", [(64, 4, 1), (128, 4, 1), (128, 8, 40), (64, 8, 700), (128, 16, 2300)])
def test_decode(stlib, D, Hq, n, size):
    """One key, of any sign; keys of one stage and of both streams; and of several runs."""
    Hkv = 2
    pool = stlib.Pool(n_layers=1, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, n_blocks=200, max_seqs=2, kv_bits=4)
    k, v = drawn(n, Hkv, D, seed=1).bfloat16(), drawn(n, Hkv, D, seed=2).bfloat16()
    q = (drawn(1, 1, Hq, D, seed=n) * size).bfloat16()
    q[0, 0, 1] = (-q[0, 0, 0].float()).bfloat16()  # the scores of the head beside it, negative
    s = pool.seq_create()
    pool.append_kv([s], k[None, None].cuda(), v[None, None].cuda())
    o, lse = pool.decode_attn([s], q.cuda())
    pool.sync()
    check_huge(o[0, 0], lse[0, 0], q[0, 0], held(k), held(v), f"size {size}")


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("order", ["rising", "falling", "drawn"])
def test_scores_that_rise_and_fall(stlib, size, order):
    D, n = 128, 1500
    pool = stlib.Pool(n_layers=1, n_q_heads=4, n_kv_heads=1, head_dim=D, n_blocks=128, max_seqs=2, kv_bits=4)
    q, k = drawn(1, 1, 4, D, seed=3), drawn(n, 1, D, seed=4)
    v = drawn(n, 1, D, seed=5).bfloat16()
    by = (k[:, 0] @ q[0, 0, 0]).argsort(descending=order == "falling")
    k = (k[by] if order != "drawn" else k).bfloat16()
    q = (q * size).bfloat16()
    s = pool.seq_create()
    pool.append_kv([s], k[None, None].cuda(), v[None, None].cuda())
    o, lse = pool.decode_attn([s], q.cuda())
    pool.sync()
    check_huge(o[0, 0], lse[0, 0], q[0, 0], held(k), held(v), f"size {size}")


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("n,T", [(0, 1), (0, 9), (0, 70), (400, 3), (2500, 40)])
def test_prefill(stlib, n, T, size):
    D, Hq = 128, 8
    pool = stlib.Pool(n_layers=1, n_q_heads=Hq, n_kv_heads=1, head_dim=D, n_blocks=200, max_seqs=2, kv_bits=4)
    k, v = drawn(n + T, 1, D, seed=6).bfloat16(), drawn(n + T, 1, D, seed=7).bfloat16()
    q = (drawn(1, T, Hq, D, seed=8) * size).bfloat16()
    s = pool.seq_create()
    if n:
        pool.append_kv([s], k[None, None, :n].contiguous().cuda(), v[None, None, :n].contiguous().cuda())
    o, lse = pool.merge(s, q.cuda(), k[None, n:].contiguous().cuda(), v[None, n:].contiguous().cuda())
    pool.sync()
    kk, vv = held(k), held(v)
    for t in sorted({0, T // 3, T // 2, T - 1}):
        check_huge(o[0, t], lse[0, t], q[0, t], kk[:n + t + 1], vv[:n + t + 1], f"size {size} row {t}")


def test_unlike_rows_and_ordinary_ones_together(stlib):
    """Heads from 2^-100 to 2^100 of an ordinary row, each as if alone."""
    D, Hq, n = 128, 16, 900
    pool = stlib.Pool(n_layers=1, n_q_heads=Hq, n_kv_heads=1, head_dim=D, n_blocks=80, max_seqs=2, kv_bits=4)
    k, v = drawn(n, 1, D, seed=9).bfloat16(), drawn(n, 1, D, seed=10).bfloat16()
    q = (drawn(1, 1, Hq, D, seed=11) * 2.0 ** torch.linspace(-100, 100, Hq).round().view(1, 1, Hq, 1)).bfloat16()
    s = pool.seq_create()
    pool.append_kv([s], k[None, None].cuda(), v[None, None].cuda())
    o, lse = pool.decode_attn([s], q.cuda())
    pool.sync()
    check_huge(o[0, 0], lse[0, 0], q[0, 0], held(k), held(v))
