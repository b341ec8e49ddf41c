"""The calls over 8-bit caches and pages on the GPU: what the header states beyond the ordinary cases -- the longest paths,
ranges that hold nothing, nodes, codes and scales that must not reach other results."""
import numpy as np
import pytest
import torch

import quant_helpers as qh
from paper_2605_07243_b200 import binding as sb
from test_gpu_quant import append_case, check, i32, make, same_cache, tree_of

pytestmark = pytest.mark.gpu

KERNELS = [(2, 2, 2, 20), (6, 8, 2, 50)]     # sequences, KV heads, heads of each, nodes: 16-row kernel, tcgen05 kernel


# ---- append ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("block,depth", [(16, 32), (16, 31), (128, 15), (64, 32)])
def test_append_paths_as_long_as_they_come(block, depth):
    """Paths of up to 33 nodes, more than a warp has lanes: every unit reads entries that other lanes have brought in."""
    layers, P = 6, [0, 5, 31, 100, 17, 64]
    N = [128, 40, depth + 1, 90, 128, 1]
    rng, cache, offs, (k, v) = append_case(71, P, N, layers=layers, D=64, block=block, page_size=128)
    paths = [sorted(rng.choice(n, size=min(n, depth + 1), replace=False).tolist()) for n in N]
    table = [p + [-1] * (depth + 1 - len(p)) for p in paths]
    kv = cache.gpu(sb)
    start = [t.clone() for t in (kv.k_codes, kv.v_codes, kv.k_scale, kv.v_scale)]
    want = qh.append_reference(cache, k.double().numpy(), v.double().numpy(), offs, P, paths)
    kg, vg = k.cuda(), v.cuda()
    args = dict(max_rows=depth + 1, path_nodes=i32(table), accept_len=i32([len(p) - 1 for p in paths]), max_depth=depth)
    for _ in range(10):
        for t, was in zip((kv.k_codes, kv.v_codes, kv.k_scale, kv.v_scale), start):
            t.copy_(was)
        new_len, status = sb.sb_kv_append_quant(kv, kg, vg, i32(offs), i32(P), **args)
        assert status.cpu().tolist() == [0] * len(P) and new_len.cpu().tolist() == want
        same_cache(kv, cache)


# ---- pages ----------------------------------------------------------------------------------------------------------------

def test_pages_reserve_of_an_empty_range_asks_for_nothing():
    """[20, 20) holds no position: the slot takes no page, is no writer of the page that it shares, and is served by a full pool."""
    pool = sb.PagePool.empty(4, 4, 4, 16)
    copies = sb.PageCopies.empty(2)
    state = lambda: [t.cpu().tolist() for t in (pool.page_table, pool.held, pool.refs)]   # noqa: E731
    assert sb.sb_pages_reserve(pool, i32([0]), i32([0]), i32([20]), copies).tolist() == [0]
    assert sb.sb_pages_fork(pool, i32([0]), i32([1]), i32([20])).tolist() == [0]
    before = state()
    assert before[0][1][:2] == [0, 1] and before[2] == [2, 2, 0, 0]
    for at in (20, 16, 1, 0):
        assert sb.sb_pages_reserve(pool, i32([1]), i32([at]), i32([at]), copies).tolist() == [0]
        assert state() == before and copies.count.item() == 0 and copies.src.tolist() == [-1, -1]
    assert sb.sb_pages_reserve(pool, i32([2]), i32([0]), i32([32]), copies).tolist() == [0]      # the pool is full
    before = state()
    assert sb.sb_pages_reserve(pool, i32([1]), i32([20]), i32([20]), copies).tolist() == [0]
    assert sb.sb_pages_reserve(pool, i32([1, 0]), i32([20, 20]), i32([20, 21]), copies).tolist() == [0, 7]
    assert state() == before and copies.count.item() == 0
    assert sb.sb_pages_release(pool, i32([2]), i32([0])).tolist() == [0]
    # slot 0 writes a page that slot 1 goes on holding: it gets one of its own
    assert sb.sb_pages_reserve(pool, i32([1, 0]), i32([20, 20]), i32([20, 21]), copies).tolist() == [0, 0]
    assert copies.count.item() == 1 and copies.src.tolist() == [1, -1] and copies.dst.tolist() == [2, -1]
    table, held, refs = state()
    assert table[0] == [0, 2, -1, -1] and table[1] == [0, 1, -1, -1] and held == [2, 2, 0, 0] and refs == [2, 1, 1, 0]


# ---- attention ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("batch,H,G,n", KERNELS)
@pytest.mark.parametrize("num_splits", [0, 1])
@pytest.mark.parametrize("log_v", [-12, -30, 20])
@pytest.mark.parametrize("gap", [0.0, 6.0, 9.0])
def test_attention_nodes_far_above_the_prefix_keep_its_share(batch, H, G, n, num_splits, log_v, gap):
    """Every node's score of itself lies `gap` above the others, and values are small or large: the prefix keeps its weight."""
    P = [[700, 0, 77, 513][b % 4] for b in range(batch)]
    cache, parents, q, k, v = make(74, P, [n] * batch, H=H, G=G, D=64, v_mag=2.0 ** log_v)
    v = (v.float() * 2.0 ** log_v).bfloat16()
    cache.scales[0][:] *= 2.0 ** -6                                     # prefix scores near zero
    cache.scales[1][:] = 2.0 ** (log_v - 6)
    q = torch.ones_like(q)
    k = torch.full_like(k, gap / 8)
    check(cache, P, parents, q, k, v, num_splits=num_splits)


@pytest.mark.parametrize("batch,H,G,n", KERNELS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(70, 0), (70, 5), (33, 130), (1, 1)])
def test_attention_nan_codes_before_the_window_do_not_matter(batch, H, G, n, D, window, sinks):
    """Rows between the sinks and the window of the root hold e4m3's NaN: no node sees them."""
    P = [[300, 200, 77, 513][b % 4] for b in range(batch)]
    cache, parents, q, k, v = make(73, P, [n] * batch, H=H, G=G, D=D, block=32)
    want, wlse = check(cache, P, parents, q, k, v, window=window, sinks=sinks)
    for b in range(batch):
        rows = [cache.row(b, j) for j in range(sinks, max(sinks, P[b] - window + 1))]
        for c in cache.codes:
            c[0, rows] = 0x7F + 0x80 * (np.arange(H * D).reshape(H, D) & 1)
    out, lse, status = sb.sb_tree_attention_quant(cache.gpu(sb), tree_of(P, parents, q.shape[1]), q.cuda(), k.cuda(), v.cuda(), window=window, sinks=sinks)
    assert status.tolist() == [0] * batch
    assert torch.equal(out, want) and torch.equal(lse, wlse)


@pytest.mark.parametrize("batch,H,G,n", KERNELS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("log_f", [6, 12, 16, 40, 100])
@pytest.mark.parametrize("which", ["k", "v", "both"])
def test_attention_large_finite_nodes_change_only_the_nodes_that_see_them(batch, H, G, n, D, log_f, which):
    """Leaves 2^log_f times larger than the other nodes.  Nobody but a leaf itself sees it: the others' results stay as they
    are with ordinary leaves, within the bound that counts their visible keys alone."""
    P = [[300, 0, 77, 513][b % 4] for b in range(batch)]
    cache, parents, q, k, v = make(72, P, [n] * batch, H=H, G=G, D=D)
    large = np.zeros(q.shape[0], bool)
    for b in range(batch):
        leaves = [i for i in range(n) if i not in parents[b]]
        large[[b * n + i for i in leaves[::2]]] = True
    f = torch.from_numpy(np.where(large, 2.0 ** log_f, 1.0)).float()[:, None, None]
    k2 = (k.float() * f).bfloat16() if which != "v" else k
    v2 = (v.float() * f).bfloat16() if which != "k" else v
    out, lse = check(cache, P, parents, q, k2, v2)
    if H == 8:      # the tcgen05 kernel keeps a row's arithmetic to itself: not a bit changes
        want, wlse = check(cache, P, parents, q, k, v)
        others = torch.from_numpy(~large).cuda()
        assert torch.equal(out[others], want[others]) and torch.equal(lse[others], wlse[others])
