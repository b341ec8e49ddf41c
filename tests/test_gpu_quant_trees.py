"""Tree attention over a KV cache in 8 bits, on the GPU: batches with more than 64 tiles of 16 rows, which the tcgen05 kernel
serves, beside small ones; scores that outgrow the running reference; what a call must not touch."""
import numpy as np
import pytest
import torch

import quant_helpers as qh
from paper_2605_07243_b200 import binding as sb
from test_gpu_quant import check, i32, make, tree_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P,N", [([0, 1, 127, 128], [33, 40, 17, 128]), ([700, 129, 255], [65, 16, 48]), ([64, 65, 63, 300, 1], [1, 60, 0, 31, 97])])
@pytest.mark.parametrize("page_size,block", [(0, 32), (16, 16), (128, 64)])
def test_trees_lengths_and_layouts(P, N, D, page_size, block):
    cache, parents, q, k, v = make(51, P, [max(n, 1) for n in N], H=8, G=2, D=D, page_size=page_size, block=block)
    if 0 in N:
        at = N.index(0)                        # a sequence without nodes
        keep = np.ones(q.shape[0], bool)
        keep[sum(max(n, 1) for n in N[:at])] = False
        parents[at], q, k, v = [], q[keep], k[keep], v[keep]
    check(cache, P, parents, q, k, v)


@pytest.mark.parametrize("H,G", [(8, 1), (5, 7), (2, 16), (33, 1)])
def test_trees_head_layouts(H, G):
    P, N = [200, 77], [70, 64]
    cache, parents, q, k, v = make(52, P, N, H=H, G=G, D=64)
    check(cache, P, parents, q, k, v)


@pytest.mark.parametrize("num_splits", [1, 2, 3, 8, 40])
def test_trees_any_number_of_chunks(num_splits):
    P, N = [513, 90], [40, 70]
    cache, parents, q, k, v = make(53, P, N, H=8, G=2)
    check(cache, P, parents, q, k, v, num_splits=num_splits)


@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 1), (20, 4), (100, 64), (100, 130), (1000, 4), (64, 600)])
def test_trees_window_and_sinks(window, sinks):
    P, N = [520, 130, 0], [60, 128, 33]
    cache, parents, q, k, v = make(54, P, N, H=8, G=1, D=64)
    check(cache, P, parents, q, k, v, window=window, sinks=sinks)


@pytest.mark.parametrize("parents", [[list(range(-1, 127))], [[-1] + [0] * 127], [[-1] * 50]])
@pytest.mark.parametrize("window", [0, 20])
def test_trees_chains_stars_and_forests(parents, window):
    parents = parents * 2
    cache, _, q, k, v = make(55, [70, 150], None, H=17, G=1, D=64, parents=parents)
    check(cache, [70, 150], parents, q, k, v, window=window, sinks=2 if window else 0)


def test_trees_queries_of_the_last_nodes():
    P, N = [100, 400], [128, 70]
    cache, parents, q, k, v = make(56, P, N, H=8, G=4, D=64)
    check(cache, P, parents, q, k, v, q_begin=[3, 50])
    check(cache, P, parents, q, k, v, q_begin=[128, 0], scale=0.3)      # the first sequence has no query


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("spread", [0.0, 6.0])
def test_trees_scales_of_very_different_size(spread, D):
    P, N = [400, 129], [50, 64]
    cache, parents, q, k, v = make(57, P, N, H=8, G=2, D=D, block=16, page_size=16, scale_spread=spread)
    cache.scales[0][:] = 2.0 ** np.clip(np.log2(cache.scales[0]), -10, -7)  # keys stay ordinary
    check(cache, P, parents, q, k, v)


@pytest.mark.parametrize("mag", [2.0 ** -40, 2.0 ** 30])
def test_trees_small_and_large_values(mag):
    cache, parents, q, k, v = make(58, [300, 200], [50, 60], H=8, G=2, v_mag=mag)
    check(cache, [300, 200], parents, q, k, (v.float() * mag).bfloat16())


def test_trees_queries_of_any_magnitude_and_scales_that_are_no_powers_of_two():
    P, N = [150, 260], [40, 70]
    cache, parents, q, k, v = make(59, P, N, H=8, G=4)
    f = q.float()
    f[:, 0] *= 2.0 ** -100
    f[:, 1] *= 2.0 ** 6
    f[:, 2] = 0
    f[:, 3, 1:] *= 2.0 ** -12
    rng = np.random.default_rng(6)
    for s in cache.scales:
        s *= rng.uniform(0.6, 1.4, size=s.shape)
        s[:] = s.astype(np.float32)
    cache.scales[0][:] = (cache.scales[0] * 2.0 ** -6).astype(np.float32)
    check(cache, P, parents, f.bfloat16(), k, v)


SMALL, LARGE = (3, 2, 1), (128, 1, 18)    # sequences, heads per KV head, nodes: 16-row kernel, tcgen05 kernel


@pytest.mark.parametrize("batch,G,n", [SMALL, LARGE])
@pytest.mark.parametrize("k_scale", [0.0, 2.0 ** -126, 2.0 ** -100, 1.0])
@pytest.mark.parametrize("q_mag", [0.0, 2.0 ** -120, 2.0 ** -20])
def test_products_that_underflow_leave_invisible_keys_invisible(batch, G, n, k_scale, q_mag):
    """Scores of nought: the result is the mean of the visible values, whatever lies behind the prefix."""
    P = [[100, 1, 17, 63][b % 4] for b in range(batch)]
    cache, parents, q, k, v = make(60, P, [n] * batch, H=1, G=G, D=64)
    cache.scales[0][:] = k_scale
    cache.codes[0][:] &= 0x87 if k_scale == 1.0 else 0xFF     # subnormal codes
    check(cache, P, parents, (q.float() * q_mag).bfloat16(), (k.float() * 0).bfloat16(), v)


@pytest.mark.parametrize("batch,G,n", [SMALL, LARGE])
@pytest.mark.parametrize("log_gap", [20, 130, 300, 2000])
def test_one_key_far_above_the_others_at_any_place(batch, G, n, log_gap):
    """Key 5 b + 3 of sequence b has a score 2^log_gap times above the others', wherever it lies in a step of the kernel."""
    D, P = 64, [700] * batch
    cache, parents, q, k, v = make(61, P, [n] * batch, H=1, G=G, D=D)
    cache.codes[0][:] = (cache.codes[0] & 0x80) | 0x10         # +-2^-5
    cache.scales[0][:] = 2.0 ** -3
    value = log_gap * np.log(2.0) / np.sqrt(D) * 8             # of each element, in units of the scale
    for b in range(batch):
        r = cache.row(b, 5 * b + 3)
        cache.codes[0][0, r] = qh.e4m3_codes(min(value, 448.0))
        if value > 448.0:
            cache.scales[0][0, r // cache.block] *= 2.0 ** np.ceil(np.log2(value / 448.0))
    check(cache, P, parents, torch.ones_like(q), k, v)


@pytest.mark.parametrize("batch,G,n", [SMALL, LARGE])
@pytest.mark.parametrize("order", ["rising", "falling", "late"])
@pytest.mark.parametrize("num_splits", [0, 1, 4])
def test_scores_that_outgrow_the_reference_again_and_again(batch, G, n, order, num_splits):
    D, length = 64, 500
    cache, parents, q, k, v = make(62, [length] * batch, [n] * batch, H=1, G=G, D=D)
    step = {"rising": np.arange(length) / 20.0, "falling": (length - np.arange(length)) / 20.0,
            "late": np.where(np.arange(length) < 400, -20.0, np.arange(length) / 100.0)}[order]
    cache.scales[0][:] = 1.0
    for b in range(batch):
        cache.codes[0][0, [cache.row(b, j) for j in range(length)]] = qh.e4m3_codes(step)[:, None, None]
    check(cache, [length] * batch, parents, torch.ones_like(q), (k.float() * 0.1).bfloat16(), v, num_splits=num_splits)


def test_trees_queries_and_nodes_that_are_not_finite():
    """A bad query row is NaN alone; a bad node of K or V makes the nodes that see it NaN; the other rows stay."""
    P, N = [300, 64], [64, 90]
    cache, parents, q, k, v = make(63, P, N, H=8, G=2)
    want, wlse = check(cache, P, parents, q, k, v)
    q2, k2, v2 = q.clone(), k.clone(), v.clone()
    q2[5, 3, 7], q2[70, 0, 0] = float("nan"), float("inf")
    k2[20, 1, 3], v2[64 + 33, 6, 0] = float("inf"), float("nan")
    out, lse, status = sb.sb_tree_attention_quant(cache.gpu(sb), tree_of(P, parents, 16), q2.cuda(), k2.cuda(), v2.cuda())
    assert status.cpu().tolist() == [0, 0]
    bad = np.zeros((q.shape[0], 16), bool)
    bad[5, 3] = bad[70, 0] = True
    for b, base, node, head in ((0, 0, 20, 1), (1, 64, 33, 6)):
        for i in range(N[b]):
            if node in qh.chain(parents[b], i):
                bad[base + i, 2 * head:2 * head + 2] = True
    bad = torch.from_numpy(bad).cuda()
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
    assert torch.equal(out[~bad], want[~bad]) and torch.equal(lse[~bad], wlse[~bad])


def test_trees_poisoned_blocks_and_stale_bytes():
    P, N = [200, 330], [45, 100]
    cache, parents, q, k, v = make(64, P, N, H=8, G=2, block=32, page_size=64)
    base, _ = check(cache, P, parents, q, k, v, window=70)
    for b in range(2):
        for j in range(P[b], cache.capacity):       # behind the prefix: NaN codes, as uninitialised memory has them
            for c in cache.codes:
                c[0, cache.row(b, j)] = 0x7F
        for s in cache.scales:
            for j in range(-(-P[b] // 32) * 32, cache.capacity, 32):
                s[0, cache.row(b, j) // 32] = np.nan
    kv, tree = cache.gpu(sb), tree_of(P, parents, 16)
    out, _, _ = sb.sb_tree_attention_quant(kv, tree, q.cuda(), k.cuda(), v.cuda(), window=70)
    assert torch.equal(out, base)
    for scales in (kv.k_scale, kv.v_scale):         # a poisoned block before every node's window, and without a window
        flat = scales.view(-1, 8)
        keep = flat.clone()
        flat[cache.row(0, 96) // 32, 3] = float("nan")
        out, _, _ = sb.sb_tree_attention_quant(kv, tree, q.cuda(), k.cuda(), v.cuda(), window=70)
        assert torch.equal(out, base)
        out, lse, _ = sb.sb_tree_attention_quant(kv, tree, q.cuda(), k.cuda(), v.cuda())
        assert torch.isnan(out[:45, 6:8]).all() and torch.isnan(lse[:45, 6:8]).all()
        assert not torch.isnan(out[:45, :6]).any() and not torch.isnan(out[:45, 8:]).any() and not torch.isnan(out[45:]).any()
        flat.copy_(keep)


def test_trees_bad_sequences_are_reported_and_the_others_served():
    P, N = [64] * 6, [40] * 6
    cache, parents, q, k, v = make(65, P, N, H=8, G=2)
    want, wlse, _ = sb.sb_tree_attention_quant(cache.gpu(sb), tree_of(P, parents, 16), q.cuda(), k.cuda(), v.cuda())
    bad = [list(t) for t in parents]
    bad[1][3] = 7                               # a parent after its child
    lens = [64, 64, 10 ** 6, 64, -1, 64]        # past the host bound; negative
    table = cache.table.copy()
    table[3, 0] = cache.pages + 7               # a page outside the pool
    out, lse, status = sb.sb_tree_attention_quant(cache.gpu(sb, table), tree_of(lens, bad, 16, max_prefix=64), q.cuda(), k.cuda(), v.cuda())
    assert status.cpu().tolist() == [0, 4, 5, 5, 5, 0]
    for b in (0, 5):
        assert torch.equal(out[40 * b:40 * b + 40], want[40 * b:40 * b + 40]) and torch.equal(lse[40 * b:40 * b + 40], wlse[40 * b:40 * b + 40])
    for b in (1, 2, 4):
        assert not out[40 * b:40 * b + 40].any() and not lse[40 * b:40 * b + 40].any()
    # a tree larger than announced, offsets that leave the rows, one that runs backwards
    tree = tree_of(P, parents, 16)
    tree = tree_of(P, parents, 16, node_offsets=i32([0, 40, 100, 90, 130, 170, 100000]), max_nodes=45)
    out = torch.full_like(want, 3.0)
    sb.sb_tree_attention_quant(cache.gpu(sb), tree, q.cuda(), k.cuda(), v.cuda(), out=out, status=(st := i32([9] * 6)))
    assert st.cpu().tolist()[0] in (0, 4) and st.cpu().tolist()[1:3] == [4, 4] and st.cpu().tolist()[5] == 4
    assert torch.equal(out[:40], want[:40])


@pytest.mark.parametrize("batch", [129, 200])
@pytest.mark.parametrize("n", [1, 20])
def test_batches_larger_than_the_planner_sorts(batch, n):
    rng = np.random.default_rng(66)
    P = [int(x) for x in rng.integers(0, 200, size=batch)]
    cache, parents, q, k, v = make(66, P, [n] * batch, H=2, G=1, D=64, page_size=16, block=16)
    check(cache, P, parents, q, k, v)


@pytest.mark.parametrize("num_splits", [0, 3])
def test_trees_write_only_their_rows_and_are_stable_under_replay(num_splits):
    P, N = [300, 100, 210], [90, 33, 128]
    cache, parents, q, k, v = make(67, P, N, H=8, G=2)
    kv, tree = cache.gpu(sb), tree_of(P, parents, 16)
    total, pad = q.shape[0], 4096
    qg, kg, vg = q.cuda(), k.cuda(), v.cuda()
    want, wlse, _ = sb.sb_tree_attention_quant(kv, tree, qg, kg, vg, num_splits=num_splits)
    outb = torch.full((2 * pad + want.numel(),), 7.0, dtype=torch.bfloat16, device="cuda")
    lseb = torch.full((2 * pad + wlse.numel(),), 7.0, dtype=torch.float32, device="cuda")
    need = max(256, sb.sb_tree_attention_quant_workspace_bytes(kv, tree, total, num_splits=num_splits))
    wsb = torch.full((2 * pad + need,), 0x5A, dtype=torch.uint8, device="cuda")
    args = dict(out=outb[pad:-pad].view_as(want), lse=lseb[pad:-pad].view_as(wlse), workspace=wsb[pad:pad + need],
                status=torch.empty(3, dtype=torch.int32, device="cuda"), num_splits=num_splits)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            sb.sb_tree_attention_quant(kv, tree, qg, kg, vg, **args)
            sb.sb_tree_attention_quant(kv, tree, qg, kg, vg, **args)     # the workspace again at once
    for _ in range(10):
        args["out"].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(args["out"], want) and torch.equal(args["lse"], wlse)
    for buf, val in ((outb, 7.0), (lseb, 7.0)):
        assert (buf[:pad] == val).all() and (buf[-pad:] == val).all()
    assert (wsb[:pad] == 0x5A).all() and (wsb[pad + need:] == 0x5A).all()


def test_calls_on_two_streams_at_once():
    P, N = [300, 100], [90, 33]
    cache, parents, q, k, v = make(68, P, N, H=8, G=2)
    kv, tree = cache.gpu(sb), tree_of(P, parents, 16)
    small = tree_of(P, [t[:1] for t in parents], 16)
    qg, kg, vg = q.cuda(), k.cuda(), v.cuda()
    q1, k1, v1 = (x[[0, 90]].contiguous() for x in (qg, kg, vg))
    want = [sb.sb_tree_attention_quant(kv, tree, qg, kg, vg, num_splits=3)[0], sb.sb_tree_attention_quant(kv, small, q1, k1, v1)[0]]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for s, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[s].append(sb.sb_tree_attention_quant(kv, tree, qg, kg, vg, num_splits=3)[0] if s == 0 else
                              sb.sb_tree_attention_quant(kv, small, q1, k1, v1)[0])
    torch.cuda.synchronize()
    for s in range(2):
        assert all(torch.equal(x, want[s]) for x in got[s])


def test_the_checked_build_finds_no_access_out_of_bounds():
    """Attention of every kernel, writes of both forms and the pages' calls, with every index checked."""
    with sb.build_variant("checked"):
        sb.sb_checked_violations()   # clear
        for P, N, H, G, D in (([300, 100, 0], [90, 33, 128], 8, 2, 128), ([129, 40], [1, 3], 2, 4, 64), ([700], [64], 8, 4, 64)):
            cache, parents, q, k, v = make(69, P, N, H=H, G=G, D=D, page_size=16, block=16)
            for kw in (dict(), dict(window=33, sinks=4), dict(num_splits=5)):
                check(cache, P, parents, q, k, v, **kw)
            kv = cache.gpu(sb)
            offs = np.concatenate([[0], np.cumsum([min(n, 3) for n in N])])
            rows = int(offs[-1])
            sb.sb_kv_append_quant(kv, k[:rows].cuda(), v[:rows].cuda(), i32(offs), i32(P), max_rows=3)
            sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32(np.concatenate([[0], np.cumsum(N)])), i32([0] * len(P)), max_rows=max(N))
        pool = qh.Pool(4, 8, 20, 16)
        gpu = pool.gpu(sb)
        copies = sb.PageCopies.empty(20)
        sb.sb_pages_reserve(gpu, i32([0, 1]), i32([0, 0]), i32([50, 16]), copies)
        sb.sb_pages_fork(gpu, i32([0, 1]), i32([2, 3]), i32([33, 16]))
        sb.sb_pages_reserve(gpu, i32([2]), i32([33]), i32([70]), copies)
        data = torch.zeros(20, 64, dtype=torch.float32, device="cuda")
        sb.sb_pages_copy(sb.PageArrays([data], n_layers=1, num_pages=20), copies)
        sb.sb_pages_release(gpu, i32([0]), i32([0]))
        sb.sb_pages_compact(gpu, copies)
        torch.cuda.synchronize()
        assert sb.sb_checked_violations() == 0


def test_pages_wishes_beyond_32_bits_are_refused():
    """1040 empty slots that ask for 2^21 pages each of a pool of ten."""
    slots, most = 1040, 1 << 21
    pool = sb.PagePool(16, torch.empty(slots, most, dtype=torch.int32, device="cuda"), torch.zeros(slots, dtype=torch.int32, device="cuda"),
                       torch.zeros(10, dtype=torch.int32, device="cuda"))
    copies = sb.PageCopies.empty(slots)
    want = [most * 16] * slots
    want[7] = 0
    status = sb.sb_pages_reserve(pool, i32(range(slots)), i32([0] * slots), i32(want), copies)
    assert status.cpu().tolist() == [7 if i != 7 else 0 for i in range(slots)]
    assert not pool.held.any() and not pool.refs.any() and copies.count.item() == 0


def test_rows_behind_the_last_sequence_stay_as_they_are():
    for P, N, H in (([40, 0], [1, 2], 2), ([300, 100], [90, 33], 8)):
        cache, parents, q, k, v = make(70, P, N, H=H, G=2)
        total = q.shape[0]
        want, wlse = check(cache, P, parents, q, k, v)
        more = torch.cat([q, q[:5]]).cuda()
        out, lse = torch.full_like(more, 3.0), torch.full(more.shape[:2], 3.0, device="cuda")
        for num_splits in (0, 11):
            sb.sb_tree_attention_quant(cache.gpu(sb), tree_of(P, parents, 2 * H), more, k.cuda(), v.cuda(), out=out, lse=lse, num_splits=num_splits,
                                       q_offsets=i32([0, N[0]]))
            assert (out[total:] == 3.0).all() and (lse[total:] == 3.0).all()
            if num_splits == 0:
                assert torch.equal(out[:total], want) and torch.equal(lse[:total], wlse)
