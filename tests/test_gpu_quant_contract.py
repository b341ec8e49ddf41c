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


@pytest.mark.parametrize("batch,H,G,n", KERNELS)
@pytest.mark.parametrize("log_gap", [6, 12])
def test_attention_blocks_of_small_scale_count_beside_large_ones(batch, H, G, n, log_gap):
    """Every second block has a V scale 2^log_gap times the others' and codes of nought, so that the result is the share of the
    small blocks alone.  A probability times its V scale is off by 2^-11 of itself or, below fp16's normal range, by 2^-25 of the largest
    probability times the largest scale; half the outputs' last bit comes on top."""
    P = [[320, 160, 64, 512][b % 4] for b in range(batch)]
    D = 64
    cache, parents, q, k, v = make(75, P, [n] * batch, H=H, G=G, D=D, block=16, page_size=16)
    cache.scales[1][:] = 2.0 ** -8
    for b in range(batch):
        for j in range(0, P[b], 32):
            r = cache.row(b, j)
            cache.scales[1][0, r // 16] = 2.0 ** (log_gap - 8)
            cache.codes[1][0, r:r + 16] = 0
    v = (v.float() * 0).bfloat16()
    out, lse, status = sb.sb_tree_attention_quant(cache.gpu(sb), tree_of(P, parents, H * G), q.cuda(), k.cuda(), v.cuda())
    assert status.tolist() == [0] * batch
    out = out.double().cpu().numpy()
    for b in range(batch):
        rows = [cache.row(b, j) for j in range(P[b])]
        kk, vv = cache.values(0, 0, b, P[b]), cache.values(1, 0, b, P[b])
        scale_v = cache.scales[1][0, np.asarray(rows) // 16]
        for i in range(n):
            at = b * n + i
            seen = qh.chain(parents[b], i)
            for h in range(H * G):
                qq = q[at, h].double().numpy() / np.sqrt(D)
                s = np.concatenate([kk[:, h // G] @ qq, k[[b * n + a for a in seen], h // G].double().numpy() @ qq])
                p = np.exp(s - s.max())
                weight = np.abs(vv[:, h // G] / scale_v[:, h // G, None])
                # scores: fp32 sums of exact products, with Q to 2^-18 of its row's largest element
                ds = 2.0 ** -18 * (np.abs(kk[:, h // G]).sum(1).max() * np.abs(qq).max())
                per = p[:P[b]] * scale_v[:, h // G]
                tol = (np.maximum(per * 2.0 ** -11, 2.0 ** -25 * p.max() * scale_v[:, h // G].max()) + 2 * ds * per) @ weight / p.sum()
                exact = p[:P[b]] @ vv[:, h // G] / p.sum()
                assert (np.abs(out[at, h] - exact) <= tol + np.abs(exact) * (2.0 ** -8 + 2 * ds) + 1e-30).all()


def test_attention_every_status_of_malformed_offsets():
    P, N = [64] * 6, [40] * 6
    cache, parents, q, k, v = make(65, P, N, H=8, G=2)
    want, wlse, _ = sb.sb_tree_attention_quant(cache.gpu(sb), tree_of(P, parents, 16), q.cuda(), k.cuda(), v.cuda())
    offsets = [0, 40, 100, 90, 130, 170, 100000]      # 40 nodes; 60, more than announced; -10; 40 and 40 across the trees; past the rows
    tree = tree_of(P, parents, 16, node_offsets=i32(offsets), max_nodes=45)
    all_parents = [p for t in parents for p in t]
    assert any(p >= i for i, p in enumerate(all_parents[90:130])) and any(p >= i for i, p in enumerate(all_parents[130:170]))
    out, lse = torch.full_like(want, 3.0), torch.full_like(wlse, 3.0)
    _, _, st = sb.sb_tree_attention_quant(cache.gpu(sb), tree, q.cuda(), k.cuda(), v.cuda(), out=out, lse=lse)
    assert st.tolist() == [0, 4, 4, 4, 4, 4]
    assert torch.equal(out[:40], want[:40]) and torch.equal(lse[:40], wlse[:40])
    assert (out[40:90] == 3.0).all() and (lse[40:90] == 3.0).all()        # nobody's rows
    assert not out[90:170].any() and not lse[90:170].any()                # rows of sequences 3 and 4, whose trees are none
    assert (out[170:] == 3.0).all() and (lse[170:] == 3.0).all()


@pytest.mark.parametrize("P,N,H", [([40, 0], [1, 2], 2), ([300, 100], [90, 33], 8)])
@pytest.mark.parametrize("num_splits", [0, 11])
def test_attention_serves_its_rows_beside_others_with_any_number_of_chunks(P, N, H, num_splits):
    cache, parents, q, k, v = make(70, P, N, H=H, G=2)
    total = q.shape[0]
    want, wlse = check(cache, P, parents, q, k, v, num_splits=num_splits)
    more = torch.cat([q, q[:5]]).cuda()
    out, lse = torch.full_like(more, 3.0), torch.full(more.shape[:2], 3.0, device="cuda")
    sb.sb_tree_attention_quant(cache.gpu(sb), tree_of(P, parents, 2 * H), more, k.cuda(), v.cuda(), out=out, lse=lse, num_splits=num_splits,
                               q_offsets=i32([0, N[0]]))
    assert (out[total:] == 3.0).all() and (lse[total:] == 3.0).all()
    assert torch.equal(out[:total], want) and torch.equal(lse[:total], wlse)


# ---- together -------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n", [1, 40])
def test_a_step_of_all_calls_replays_from_a_graph(n):
    """Fork, reserve, copy, attend, append, release and compact as one graph: replayed from the same state it leaves, bit for bit, what the
    calls leave one by one; replayed on other inputs, what they leave on those."""
    H, G, D, ps, block, slots, num, layers = 4, 4, 64, 32, 16, 6, 60, 2
    rng = np.random.default_rng(76)
    pool = sb.PagePool.empty(slots, 10, num, ps)
    codes = [torch.zeros(layers, num, ps, H, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones(layers, num, ps // block, H, device="cuda") for _ in range(2)]
    kv = sb.QuantCache(codes[0], codes[1], scales[0], scales[1], H, D, block, page_size=ps, page_table=pool.page_table, n_layers=layers)
    arrays = sb.PageArrays(codes + scales, n_layers=layers, num_pages=num)
    copies = [sb.PageCopies.empty(num) for _ in range(2)]
    length = i32([0] * slots)
    # a prompt in slots 0 and 1
    sb.sb_pages_reserve(pool, i32([0, 1]), i32([0, 0]), i32([100, 75]), copies[0])
    rows = [qh.bf16_of(rng.normal(size=(layers, 175, H, D))).cuda() for _ in range(2)]
    new, status = sb.sb_kv_append_quant(kv, rows[0], rows[1], i32([0, 100, 175, 175, 175, 175, 175]), length, max_rows=100)
    assert status.tolist() == [0] * slots
    length = i32([100, 75, 75, 0, 0, 0])             # slot 2 will branch from slot 1
    offs, live = i32([n * b for b in range(slots + 1)]), i32([0, 1, 2])
    parents = [qh.random_parents(rng, n) for _ in range(slots)]
    q, k, v = (qh.bf16_of(rng.normal(size=(n * slots, h, D))).cuda() for h in (H * G, H, H))
    kl, vl = (torch.stack([x, x * 0.5]) for x in (k, v))
    path = i32([sorted(qh.chain(t, n - 1))[:4] + [-1] * (4 - min(4, len(qh.chain(t, n - 1)))) for t in parents])
    accept = (path >= 0).sum(dim=1, dtype=torch.int32) - 1
    tree = sb.QuantTree(n_q_heads=H * G, prefix_len=length, node_offsets=offs, parent=i32([p for t in parents for p in t]), max_nodes=n, max_prefix=200)
    slots_of = [i32([1]), i32([2]), i32([75])]
    grown = i32([104, 79, 79])
    gone, none = i32([0]), i32([0])
    state = [pool.page_table, pool.held, pool.refs] + codes + scales
    start = [t.clone() for t in state]

    def step():
        out = [sb.sb_pages_fork(pool, *slots_of),
               sb.sb_pages_reserve(pool, live, length[:3], grown, copies[0])]
        sb.sb_pages_copy(arrays, copies[0])
        out += sb.sb_tree_attention_quant(kv, tree, q, k, v, layer=1, window=60, sinks=4, num_splits=2)
        out += sb.sb_kv_append_quant(kv, kl, vl, offs, length, max_rows=4, path_nodes=path, accept_len=accept, max_depth=3)
        out += [sb.sb_pages_release(pool, gone, none), sb.sb_pages_compact(pool, copies[1])]
        sb.sb_pages_copy(arrays, copies[1])
        return out

    def run(fn):
        for t, was in zip(state, start):
            t.copy_(was)
        out = fn()
        torch.cuda.synchronize()
        return [t.clone() for t in state + list(out) + [copies[1].src, copies[1].dst]]

    want = run(step)
    assert want[len(state)].tolist() == [0] and want[len(state) + 1].tolist() == [0, 0, 0]
    assert want[len(state) + 4].tolist()[:3] == [0, 0, 0] and want[len(state) + 6].tolist()[:3] == [0, 0, 0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            held = step()
    torch.cuda.current_stream().wait_stream(side)

    def replay():
        g.replay()
        return held

    for _ in range(5):
        for a, b in zip(run(replay), want):
            assert torch.equal(a, b)
    q.mul_(0.5)
    kl.neg_()
    k.copy_(kl[0])
    want = run(step)
    for a, b in zip(run(replay), want):
        assert torch.equal(a, b)
