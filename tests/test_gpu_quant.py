"""The calls over a KV cache in 8 bits and over its pages, on the GPU, against plain references in 64 bits."""
import numpy as np
import pytest
import torch

import quant_helpers as qh
from paper_2605_07243_b200 import binding as sb

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def make(seed, P, N, H=2, G=4, D=128, block=64, page_size=64, layers=1, parents=None, **kw):
    rng = np.random.default_rng(seed)
    cache = qh.Cache(rng, len(P), H, D, block, page_size, max(P) + 3, layers=layers, **kw)
    parents = [qh.random_parents(rng, n) for n in N] if parents is None else parents
    total = sum(len(t) for t in parents)
    q = qh.bf16_of(rng.normal(size=(total, H * G, D)) * 1.3)
    k = qh.bf16_of(rng.normal(size=(total, H, D)))
    v = qh.bf16_of(rng.normal(size=(total, H, D)))
    return cache, parents, q, k, v


def tree_of(P, parents, n_q_heads, **kw):
    offs = np.concatenate([[0], np.cumsum([len(t) for t in parents])])
    d = dict(n_q_heads=n_q_heads, prefix_len=i32(P), node_offsets=i32(offs), parent=i32([p for t in parents for p in t]),
             max_nodes=max(1, max(len(t) for t in parents)), max_prefix=max(P))
    d.update(kw)
    return sb.QuantTree(**d)


def check(cache, P, parents, q, k, v, *, layer=0, window=0, sinks=0, num_splits=0, q_begin=None, scale=0.0, gpu=None):
    kv = cache.gpu(sb) if gpu is None else gpu
    tree = tree_of(P, parents, q.shape[1])
    kw = {}
    sel = np.arange(q.shape[0])
    if q_begin is not None:
        offs = np.concatenate([[0], np.cumsum([len(t) for t in parents])])
        sel = np.concatenate([np.arange(offs[b] + q_begin[b], offs[b + 1]) for b in range(len(P))])
        kw = dict(q_node_begin=i32(q_begin), q_offsets=i32(np.concatenate([[0], np.cumsum([len(t) - s for t, s in zip(parents, q_begin)])[:-1]])))
    qs = q[sel]
    out, lse, status = sb.sb_tree_attention_quant(kv, tree, qs.cuda(), k.cuda(), v.cuda(), layer=layer, window=window, sinks=sinks,
                                                  num_splits=num_splits, scale=scale, **kw)
    assert status.cpu().tolist() == [0] * len(P)
    ref, rlse, tol, ltol = qh.attention_reference(cache, layer, qs.double().numpy(), k.double().numpy(), v.double().numpy(), P, parents,
                                                  window, sinks, scale or None, q_begin)
    err = np.abs(out.double().cpu().numpy() - ref)
    assert (err <= tol).all(), f"out: {np.max(err / tol):.2f} of the bound, error {err.max():.2e}"
    lerr = np.abs(lse.double().cpu().numpy() - rlse)
    assert (lerr <= ltol).all(), f"lse: {np.max(lerr / ltol):.2f} of the bound, error {lerr.max():.2e}"
    return out, lse


# ---- attention ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P,N", [([0], [1]), ([1], [1]), ([15, 16, 17], [1, 1, 1]), ([31, 32, 33], [2, 1, 3]), ([63, 64, 65, 0], [1, 5, 1, 2]),
                                 ([127, 128, 129], [4, 16, 17]), ([700], [33]), ([255, 300], [127, 128])])
@pytest.mark.parametrize("page_size,block", [(0, 32), (16, 16), (64, 64), (128, 32)])
def test_attention_lengths_and_layouts(P, N, D, page_size, block):
    cache, parents, q, k, v = make(11, P, N, D=D, page_size=page_size, block=block, G=2 if max(N) > 40 else 4)
    check(cache, P, parents, q, k, v)


@pytest.mark.parametrize("H,G", [(1, 1), (3, 1), (1, 5), (2, 7), (1, 16), (8, 4)])
def test_attention_head_layouts(H, G):
    P, N = [200, 77], [9, 3]
    cache, parents, q, k, v = make(12, P, N, H=H, G=G)
    check(cache, P, parents, q, k, v)


@pytest.mark.parametrize("num_splits", [1, 2, 3, 5, 8, 11, 16, 40])
@pytest.mark.parametrize("N", [[1, 1], [40, 70]])
def test_attention_any_number_of_chunks(num_splits, N):
    P = [513, 90]  # more chunks than key blocks for the short one
    cache, parents, q, k, v = make(13, P, N, D=128)
    check(cache, P, parents, q, k, v, num_splits=num_splits)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (2, 1), (16, 0), (33, 4), (100, 64), (100, 130), (1000, 4), (64, 600)])
@pytest.mark.parametrize("P,N", [([300, 5, 0, 129], [20, 7, 3, 1]), ([520], [60])])
def test_attention_window_and_sinks(window, sinks, P, N):
    cache, parents, q, k, v = make(14, P, N, G=3)
    check(cache, P, parents, q, k, v, window=window, sinks=sinks)
    check(cache, P, parents, q, k, v, window=window, sinks=sinks, num_splits=3)


def test_attention_chain_and_star_trees_at_the_node_limit():
    P = [70, 70]
    parents = [[-1] + list(range(127)), [-1] + [0] * 127]
    cache, _, q, k, v = make(15, P, [128, 128], G=1, parents=parents)
    check(cache, P, parents, q, k, v)
    check(cache, P, parents, q, k, v, window=20, sinks=2)


def test_attention_forest_and_queries_of_the_last_nodes():
    P, parents = [100, 40], [[-1, -1, 0, 1, 2, -1, 4], [-1, 0, 0]]
    cache, _, q, k, v = make(16, P, None, parents=parents)
    check(cache, P, parents, q, k, v)
    check(cache, P, parents, q, k, v, q_begin=[3, 0])
    check(cache, P, parents, q, k, v, q_begin=[6, 3])      # the second sequence has no query
    check(cache, P, parents, q, k, v, scale=0.3)


def test_attention_reads_its_own_layer_and_strided_rows():
    P, N = [200, 333], [5, 30]
    cache, parents, q, k, v = make(17, P, N, layers=3)
    kv = cache.gpu(sb)
    outs = [check(cache, P, parents, q, k, v, layer=i, gpu=kv)[0] for i in range(3)]
    assert not torch.equal(outs[0], outs[2])
    # q, k and v as slices of one projection
    total, H, D = k.shape
    Hq = q.shape[1]
    fused = torch.zeros(total, Hq + 2 * H, D, dtype=torch.bfloat16, device="cuda")
    fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:] = q.cuda(), k.cuda(), v.cuda()
    got, _, _ = sb.sb_tree_attention_quant(kv, tree_of(P, parents, Hq), fused[:, :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:], layer=2)
    assert torch.equal(got, outs[2])


@pytest.mark.parametrize("N", [[1, 1], [50, 64]])
@pytest.mark.parametrize("spread", [0.0, 6.0])
def test_attention_scales_of_very_different_size(spread, N):
    """Neighbouring blocks whose values differ by factors of thousands: the largest must not drown the rest."""
    P = [400, 129]
    cache, parents, q, k, v = make(18, P, N, block=16, page_size=16, scale_spread=spread)
    cache.scales[0][:] = 2.0 ** np.clip(np.log2(cache.scales[0]), -10, -7)  # keys stay ordinary
    check(cache, P, parents, q, k, v)


@pytest.mark.parametrize("N", [[1], [50]])
@pytest.mark.parametrize("mag", [2.0 ** -40, 2.0 ** 30])
def test_attention_small_and_large_values(mag, N):
    cache, parents, q, k, v = make(19, [300], N, v_mag=mag)
    v = (v.float() * mag).bfloat16()
    check(cache, [300], parents, q, k, v)


@pytest.mark.parametrize("N", [1, 50])
def test_attention_scales_that_are_no_powers_of_two_and_zero_blocks(N):
    cache, parents, q, k, v = make(20, [200], [N])
    rng = np.random.default_rng(5)
    for s in cache.scales:
        s[:] = (s * (0.5 + rng.random(s.shape))).astype(np.float32)
    cache.scales[1][0, cache.row(0, 64) // 64] = 2.0 ** -100   # a block of zeros as the writer leaves it
    rows = [cache.row(0, j) for j in range(64, 128)]
    cache.codes[1][0, rows] = 0
    check(cache, [200], parents, q, k, v)


@pytest.mark.parametrize("N", [1, 40])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_queries_of_any_magnitude(N, D):
    cache, parents, q, k, v = make(21, [150], [N], D=D)
    f = q.float()
    f[:, 0] *= 2.0 ** -100
    f[:, 1] *= 2.0 ** 20
    f[:, 2] = 0
    f[:, 3, 1:] *= 2.0 ** -12
    cache.scales[0][:] *= 2.0 ** -6
    check(cache, [150], parents, f.bfloat16(), k, v)


@pytest.mark.parametrize("P,N", [([100], [7]), ([300, 64], [64, 90])])
def test_attention_nonfinite_values_in_masked_places_do_not_matter(P, N):
    """A node row, a poisoned block and stale bytes that a row does not see change nothing for it; rows that see them get
    NaN."""
    cache, parents, q, k, v = make(22, P, N)
    want, wlse = check(cache, P, parents, q, k, v)
    bad_node = len(parents[0]) - 2
    for which, val in ((0, float("nan")), (0, float("inf")), (1, float("nan")), (1, -float("inf"))):
        k2, v2 = k.clone(), v.clone()
        (k2, v2)[which][bad_node, 1, 3] = val
        out, lse, status = sb.sb_tree_attention_quant(cache.gpu(sb), tree_of(P, parents, q.shape[1]), q.cuda(), k2.cuda(), v2.cuda())
        assert status.cpu().tolist() == [0] * len(P)
        offs = 0
        for b, t in enumerate(parents):
            for i in range(len(t)):
                sees = b == 0 and bad_node in qh.chain(t, i)
                row, lrow = out[offs + i], lse[offs + i]
                G = q.shape[1] // k.shape[1]
                assert torch.equal(row[:G], want[offs + i, :G]) and torch.equal(lrow[:G], wlse[offs + i, :G])   # the other KV head
                if sees:
                    assert torch.isnan(row[G:]).all() and torch.isnan(lrow[G:]).all()
                else:
                    assert torch.equal(row[G:], want[offs + i, G:])
            offs += len(t)


@pytest.mark.parametrize("N", [1, 45])
def test_attention_poisoned_block_and_stale_bytes(N):
    P = [200]
    cache, parents, q, k, v = make(23, P, [N], block=32, page_size=64)
    base, _ = check(cache, P, parents, q, k, v, window=70)
    for j in range(200, cache.capacity):       # behind the prefix: NaN codes, as uninitialised memory has them
        for c in cache.codes:
            c[0, cache.row(0, j)] = 0x7F
    for s in cache.scales:
        s[0, cache.row(0, 224) // 32] = np.nan
    kv = cache.gpu(sb)
    tree = tree_of(P, parents, q.shape[1])
    out, _, _ = sb.sb_tree_attention_quant(kv, tree, q.cuda(), k.cuda(), v.cuda(), window=70)
    assert torch.equal(out, base)
    for which in (0, 1):                       # a poisoned block inside the prefix, before every node's window ...
        scales = (kv.k_scale, kv.v_scale)[which]
        keep = scales.clone()
        flat = scales.view(-1, 2)
        flat[cache.row(0, 96) // 32, 0] = float("nan")
        out, _, _ = sb.sb_tree_attention_quant(kv, tree, q.cuda(), k.cuda(), v.cuda(), window=70)
        assert torch.equal(out, base)
        out, lse, _ = sb.sb_tree_attention_quant(kv, tree, q.cuda(), k.cuda(), v.cuda())          # ... and without a window
        G = q.shape[1] // 2
        assert torch.isnan(out[:, :G]).all() and torch.isnan(lse[:, :G]).all() and not torch.isnan(out[:, G:]).any()
        scales.copy_(keep)


def test_attention_bad_sequences_are_reported_and_the_others_served():
    P, N = [64, 64, 64, 64, 64], [4, 4, 4, 4, 4]
    cache, parents, q, k, v = make(24, P, N)
    want, wlse, _ = sb.sb_tree_attention_quant(cache.gpu(sb), tree_of(P, parents, q.shape[1]), q.cuda(), k.cuda(), v.cuda())
    bad = [list(t) for t in parents]
    bad[1] = [-1, 0, 3, 1]                      # a parent after its child
    lens = [64, 64, 10 ** 6, 64, -1]            # past the host bound; negative
    table = cache.table.copy()
    table[3, 0] = cache.pages + 7               # a page outside the pool
    out, lse, status = sb.sb_tree_attention_quant(cache.gpu(sb, table), tree_of(lens, bad, q.shape[1], max_prefix=64), q.cuda(), k.cuda(), v.cuda())
    assert status.cpu().tolist() == [0, 4, 5, 5, 5]
    assert torch.equal(out[:4], want[:4]) and torch.equal(lse[:4], wlse[:4])
    for b in (1, 2, 4):
        assert not out[4 * b:4 * b + 4].any() and not lse[4 * b:4 * b + 4].any()


@pytest.mark.parametrize("P,N", [([40, 0], [1, 1]), ([300, 100], [90, 33])])
def test_attention_writes_only_its_rows_and_is_stable_under_replay(P, N):
    cache, parents, q, k, v = make(25, P, N)
    kv, tree = cache.gpu(sb), tree_of(P, parents, q.shape[1])
    total = q.shape[0]
    want, wlse, _ = sb.sb_tree_attention_quant(kv, tree, q.cuda(), k.cuda(), v.cuda(), num_splits=3)
    # output, log-sum-exp and workspace inside larger buffers
    pad = 4096
    outb = torch.full((2 * pad + want.numel(),), 7.0, dtype=torch.bfloat16, device="cuda")
    lseb = torch.full((2 * pad + wlse.numel(),), 7.0, dtype=torch.float32, device="cuda")
    need = sb.sb_tree_attention_quant_workspace_bytes(kv, tree, total, num_splits=3)
    wsb = torch.full((2 * pad + need,), 0x5A, dtype=torch.uint8, device="cuda")
    status = torch.empty(len(P), dtype=torch.int32, device="cuda")
    args = dict(out=outb[pad:-pad].view_as(want), lse=lseb[pad:-pad].view_as(wlse), workspace=wsb[pad:pad + need], status=status, num_splits=3)
    if need == 0:
        args["workspace"] = wsb[pad:pad + 256]
    qg, kg, vg = q.cuda(), k.cuda(), v.cuda()
    sb.sb_tree_attention_quant(kv, tree, qg, kg, vg, **args)
    assert torch.equal(args["out"], want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            sb.sb_tree_attention_quant(kv, tree, qg, kg, vg, **args)
    for _ in range(20):
        args["out"].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(args["out"], want) and torch.equal(args["lse"], wlse)
    for buf, val in ((outb, 7.0), (lseb, 7.0)):
        assert (buf[:pad] == val).all() and (buf[-pad:] == val).all()
    assert (wsb[:pad] == 0x5A).all() and (wsb[pad + max(need, 256):] == 0x5A).all()


def test_attention_offsets_past_32_bits():
    """A paged cache whose last pages start beyond 2^32 bytes."""
    H, D, ps = 8, 128, 128
    pages = (1 << 32) // (ps * H * D) + 40
    P, parents = [ps * 3 + 5], [[-1, 0, 1, 0]]
    rng = np.random.default_rng(3)
    small = qh.Cache(rng, 1, H, D, 64, ps, P[0], spare=0)
    codes = [torch.zeros(pages, ps, H, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones(pages, ps // 64, H, device="cuda") for _ in range(2)]
    ids = np.asarray([pages - 1, 0, pages - 7, pages - 3], np.int32)
    for j, page in enumerate(ids):
        for w in (0, 1):
            at = int(small.table[0, j])
            codes[w][page] = torch.from_numpy(small.codes[w].reshape(-1, ps, H, D)[at]).cuda()
            scales[w][page] = torch.from_numpy(small.scales[w].reshape(-1, ps // 64, H)[at].astype(np.float32)).cuda()
    kv = sb.QuantCache(codes[0], codes[1], scales[0], scales[1], H, D, 64, page_size=ps, page_table=torch.from_numpy(ids[None]).cuda())
    q, k, v = (qh.bf16_of(rng.normal(size=(4, h, D))) for h in (2 * H, H, H))
    check(small, P, parents, q, k, v, gpu=kv)
    # and the writer: rows that land on the last pages
    new_len, status = sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32([0, 4]), i32(P), max_rows=4)
    assert status.tolist() == [0] and new_len.tolist() == [P[0] + 4]
    qh.append_reference(small, k.double().numpy()[None], v.double().numpy()[None], [0, 4], P)
    for w in (0, 1):
        got = codes[w][int(ids[3])].cpu().numpy()
        np.testing.assert_array_equal(got, small.codes[w].reshape(-1, ps, H, D)[int(small.table[0, 3])])


def test_attention_on_a_stream_of_its_own():
    P, N = [300], [20]
    cache, parents, q, k, v = make(26, P, N)
    kv, tree = cache.gpu(sb), tree_of(P, parents, q.shape[1])
    want, _, _ = sb.sb_tree_attention_quant(kv, tree, q.cuda(), k.cuda(), v.cuda())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got, _, _ = sb.sb_tree_attention_quant(kv, tree, q.cuda(), k.cuda(), v.cuda())
    s.synchronize()
    assert torch.equal(got, want)


# ---- append ---------------------------------------------------------------------------------------------------------------

def same_cache(kv, cache):
    for w, (codes, scales) in enumerate(((kv.k_codes, kv.k_scale), (kv.v_codes, kv.v_scale))):
        np.testing.assert_array_equal(codes.cpu().numpy().reshape(cache.codes[w].shape), cache.codes[w])
        np.testing.assert_array_equal(scales.cpu().numpy().astype(np.float64).reshape(cache.scales[w].shape), cache.scales[w])


def append_case(seed, P, n, H=2, D=64, block=32, page_size=64, layers=1, mag=1.0):
    rng = np.random.default_rng(seed)
    cache = qh.Cache(rng, len(P), H, D, block, page_size, max(p + m for p, m in zip(P, n)) + 1, layers=layers)
    offs = np.concatenate([[0], np.cumsum(n)]).astype(int)
    rows = [qh.bf16_of(rng.normal(size=(layers, offs[-1], H, D)) * mag * np.exp(rng.normal(size=(1, offs[-1], 1, 1)))) for _ in range(2)]
    return rng, cache, offs, rows


@pytest.mark.parametrize("D,H", [(64, 1), (64, 3), (128, 2)])
@pytest.mark.parametrize("page_size,block", [(0, 16), (0, 128), (16, 16), (64, 32), (128, 128)])
@pytest.mark.parametrize("P,n", [([0], [1]), ([0, 31, 32, 33], [5, 1, 1, 200]), ([100, 0, 17], [0, 129, 15])])
def test_append_codes_and_scales_are_exact(D, H, page_size, block, P, n):
    _, cache, offs, (k, v) = append_case(31, P, n, H=H, D=D, block=block, page_size=page_size)
    kv = cache.gpu(sb)
    new_len, status = sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32(offs), i32(P), max_rows=max(n))
    want = qh.append_reference(cache, k.double().numpy(), v.double().numpy(), offs, P)
    assert status.cpu().tolist() == [0] * len(P) and new_len.cpu().tolist() == want
    same_cache(kv, cache)


@pytest.mark.parametrize("mag", [2.0 ** -110, 2.0 ** -20, 2.0 ** 15, 2.0 ** 60])
def test_append_scales_over_the_whole_range(mag):
    P, n = [0, 20], [40, 40]
    _, cache, offs, (k, v) = append_case(32, P, n, mag=mag)
    k[0, 3] = 0
    k[0, 32:40] = 0
    kv = cache.gpu(sb)
    sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32(offs), i32(P), max_rows=40)
    qh.append_reference(cache, k.double().numpy(), v.double().numpy(), offs, P)
    same_cache(kv, cache)


def test_append_every_bf16_magnitude_rounds_to_the_nearest_code():
    """All bf16 values within a block's range, ties among them."""
    vals = torch.arange(0x3000, 0x43E1, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)   # up to 448
    n = -(-vals.numel() // 62) * 62
    x = torch.zeros(n, dtype=torch.bfloat16)
    x[:vals.numel()] = vals
    rows = torch.cat([x.view(-1, 62), torch.full((n // 62, 1), 448.0), torch.full((n // 62, 1), -448.0)], dim=1).bfloat16()
    m = rows.shape[0]
    rows = rows.view(1, m, 1, 64)
    cache = qh.Cache(np.random.default_rng(0), 1, 1, 64, 16, 0, m)
    kv = cache.gpu(sb)
    sb.sb_kv_append_quant(kv, rows.cuda(), -rows.cuda(), i32([0, m]), i32([0]), max_rows=m)
    qh.append_reference(cache, rows.double().numpy(), -rows.double().numpy(), [0, m], [0])
    assert (cache.scales[0][0, :m // 16] == 1.0).all()
    same_cache(kv, cache)


def test_append_in_pieces_grows_the_scale_of_older_tokens():
    """Row by row with growing, equal and falling magnitudes; the older codes follow."""
    mags = [1.0, 0.01, 3.0, 3.0, 100.0, 0.5, 70000.0, 1e-3, 1.0] * 5
    _, cache, _, (k, v) = append_case(33, [3], [len(mags)], block=16, page_size=16)
    scale = torch.tensor(mags).view(1, -1, 1, 1)
    k, v = (k.float() * scale).bfloat16(), (v.float() / scale).bfloat16()
    kv = cache.gpu(sb)
    length = i32([3])
    for i in range(len(mags)):
        new, _ = sb.sb_kv_append_quant(kv, k[:, i:i + 1].cuda(), v[:, i:i + 1].cuda(), i32([0, 1]), length, max_rows=1)
        qh.append_reference(cache, k[:, i:i + 1].double().numpy(), v[:, i:i + 1].double().numpy(), [0, 1], [3 + i])
        length = new.clone()
        assert length.item() == 4 + i
    same_cache(kv, cache)


@pytest.mark.parametrize("layers", [1, 5])
def test_append_accepted_paths_of_all_layers(layers):
    P, N = [0, 31, 100, 64], [8, 40, 3, 128]
    rng, cache, offs, (k, v) = append_case(34, P, N, layers=layers, D=128)
    paths = [[0, 2, 3, 7], [0] + sorted(rng.choice(np.arange(1, 40), 8, replace=False).tolist()), [0], [0, 127]]
    max_depth = 8
    kv = cache.gpu(sb)
    table = [p + [-1] * (max_depth + 1 - len(p)) for p in paths]
    new_len, status = sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32(offs), i32(P), max_rows=9, path_nodes=i32(table),
                                            accept_len=i32([len(p) - 1 for p in paths]), max_depth=max_depth)
    want = qh.append_reference(cache, k.double().numpy(), v.double().numpy(), offs, P, paths)
    assert status.cpu().tolist() == [0] * 4 and new_len.cpu().tolist() == want
    same_cache(kv, cache)


def test_append_strided_rows_of_a_fused_projection():
    P, n = [10, 50], [7, 33]
    _, cache, offs, (k, v) = append_case(35, P, n, layers=2)
    fused = torch.zeros(2, offs[-1], 9, 64, dtype=torch.bfloat16, device="cuda")
    fused[:, :, 5:7], fused[:, :, 7:9] = k.cuda(), v.cuda()
    kv = cache.gpu(sb)
    sb.sb_kv_append_quant(kv, fused[:, :, 5:7], fused[:, :, 7:9], i32(offs), i32(P), max_rows=33)
    qh.append_reference(cache, k.double().numpy(), v.double().numpy(), offs, P)
    same_cache(kv, cache)


def test_append_nonfinite_rows_poison_their_block_only():
    P, n = [5], [60]
    _, cache, offs, (k, v) = append_case(36, P, n, block=16, page_size=16)
    k[0, 3, 1, 5] = float("nan")
    v[0, 30, 0, 0] = float("inf")
    kv = cache.gpu(sb)
    sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32(offs), i32(P), max_rows=60)
    qh.append_reference(cache, k.double().numpy(), v.double().numpy(), offs, P)
    assert np.isnan(cache.scales[0]).sum() == 1 and np.isnan(cache.scales[1]).sum() == 1
    same_cache(kv, cache)
    # a poisoned block stays poisoned when more tokens come
    more = qh.bf16_of(np.random.default_rng(1).normal(size=(1, 2, 2, 64)))
    cache.scales[0][0, cache.row(0, 64) // 16, 0] = np.nan
    kv = cache.gpu(sb)
    sb.sb_kv_append_quant(kv, more.cuda(), more.cuda(), i32([0, 2]), i32([65]), max_rows=2)
    qh.append_reference(cache, more.double().numpy(), more.double().numpy(), [0, 2], [65])
    same_cache(kv, cache)


def test_append_bad_sequences_write_nothing():
    P, n = [0, 0, 0, 0], [20, 20, 20, 20]
    _, cache, offs, (k, v) = append_case(37, P, n, page_size=32, block=16)
    table = cache.table.copy()
    table[1, 0] = cache.pages                     # page outside the pool
    before = [c.copy() for c in cache.codes]
    kv = cache.gpu(sb, table)
    lens = [cache.capacity - 19, 0, -1, 0]        # one position too many; -; negative; fine
    new_len, status = sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32(offs), i32(lens), max_rows=20)
    assert status.cpu().tolist() == [5, 5, 5, 0] and new_len.cpu().tolist() == [cache.capacity - 19, 0, -1, 20]
    rows = np.ones(cache.rows, bool)
    rows[[cache.row(3, j) for j in range(20)]] = False
    assert (kv.k_codes.cpu().numpy().reshape(before[0].shape)[:, rows] == before[0][:, rows]).all()
    # offsets out of order, more rows than announced, and paths that are none
    kv = cache.gpu(sb)
    _, status = sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32([0, 30, 20, 41, 200]), i32(P), max_rows=25)
    assert status.cpu().tolist() == [4, 4, 0, 4]
    _, status = sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32(offs), i32(P), max_rows=3, max_depth=2, accept_len=i32([1, 2, 3, 1]),
                                      path_nodes=i32([[0, 20, -1], [0, 5, 5], [0, 1, 2], [0, -3, -1]]))
    assert status.cpu().tolist() == [4, 4, 4, 4]


# ---- pages ----------------------------------------------------------------------------------------------------------------

def reserve(pool, gpu, slots, keep, new):
    copies = sb.PageCopies.empty(len(slots))
    status = sb.sb_pages_reserve(gpu, i32(slots), i32(keep), i32(new), copies)
    want, pairs = pool.reserve(slots, keep, new)
    assert status.cpu().tolist() == want
    n = copies.count.item()
    assert list(zip(copies.src.tolist()[:n], copies.dst.tolist()[:n])) == pairs
    assert copies.src.tolist()[n:] == copies.dst.tolist()[n:] == [-1] * (len(slots) - n)
    pool.same(gpu)
    return copies


def test_pages_life_of_a_few_sequences():
    pool = qh.Pool(6, 8, 20, 16)
    gpu = pool.gpu(sb)
    reserve(pool, gpu, [0, 1], [0, 0], [50, 16])
    for args in (([0, 0, 1], [2, 3, 4], [50, 33, 0]),):
        st = sb.sb_pages_fork(gpu, *(i32(a) for a in args))
        assert st.cpu().tolist() == pool.fork(*args) == [0, 0, 0]
        pool.same(gpu)
    reserve(pool, gpu, [2, 0, 3], [50, 50, 33], [51, 80, 48])    # 0 and 2 share their last page, 3 shares a page of theirs
    reserve(pool, gpu, [3], [32, ], [48])
    st = sb.sb_pages_release(gpu, i32([0, 2]), i32([17, 0]))
    assert st.cpu().tolist() == pool.release([0, 2], [17, 0])
    pool.same(gpu)
    copies, used = sb.PageCopies.empty(10), i32([0])
    st = sb.sb_pages_compact(gpu, copies, n_used=used)
    pairs, n_used = pool.compact()
    assert st.item() == 0 and used.item() == n_used and copies.count.item() == len(pairs)
    assert list(zip(copies.src.tolist(), copies.dst.tolist()))[:len(pairs)] == pairs
    pool.same(gpu)


@pytest.mark.parametrize("seed", range(6))
def test_pages_random_walk(seed):
    """Hundreds of calls on a tight pool, refused ones among them; every state equals the reference's."""
    rng = np.random.default_rng(seed)
    slots, max_pages, ps = [(40, 6, 16), (3, 200, 16), (130, 3, 64)][seed % 3]
    num = int(slots * max_pages * (0.2 + 0.4 * rng.random())) + 1
    pool = qh.Pool(slots, max_pages, num, ps)
    gpu = pool.gpu(sb)
    refused = 0
    for step in range(60):
        n = int(rng.integers(1, slots + 2))
        pick = lambda: [int(x) for x in rng.integers(-1 if rng.random() < 0.1 else 0, slots + (rng.random() < 0.1), size=n)]   # noqa: E731
        kind = rng.integers(0, 4)
        s = pick() if rng.random() < 0.5 else [int(x) for x in rng.permutation(slots)[:n]]
        n = len(s)
        held = [len(pool.rows[x]) * ps if 0 <= x < slots else 0 for x in s]
        if kind == 0:
            keep = [int(rng.integers(-1 if rng.random() < 0.05 else 0, h + 1 + (rng.random() < 0.05))) for h in held]
            st = sb.sb_pages_release(gpu, i32(s), i32(keep))
            want = pool.release(s, keep)
        elif kind == 1:
            d = pick()[:n] + [0] * max(0, n - len(pick()))
            d = (d * n)[:n]
            length = [int(rng.integers(0, h + 1 + (rng.random() < 0.05))) for h in held]
            st = sb.sb_pages_fork(gpu, i32(s), i32(d), i32(length))
            want = pool.fork(s, d, length)
        elif kind == 2:
            keep = [int(rng.integers(0, h + 1 + (rng.random() < 0.05))) for h in held]
            new = [k + int(rng.integers(-1 if rng.random() < 0.05 else 0, 3 * ps)) for k in keep]
            reserve(pool, gpu, s, keep, new)
            continue
        else:
            copies, used = sb.PageCopies.empty(num // 2 + int(rng.integers(0, 3))), i32([0])
            st = sb.sb_pages_compact(gpu, copies, n_used=used)
            pairs, n_used = pool.compact()
            m = copies.count.item()
            assert list(zip(copies.src.tolist(), copies.dst.tolist()))[:m] == pairs and used.item() == n_used
            assert copies.src.tolist()[m:] == [-1] * (copies.src.numel() - m)
            want = [0]
        assert st.cpu().tolist() == want
        refused += sum(e != 0 for e in want)
        pool.same(gpu)
    assert refused > 0 or seed % 3 == 1


def test_pages_all_holders_in_one_call_keep_one_page():
    pool = qh.Pool(5, 4, 12, 16)
    gpu = pool.gpu(sb)
    reserve(pool, gpu, [4], [0], [20])
    sb.sb_pages_fork(gpu, i32([4, 4, 4]), i32([0, 1, 2]), i32([20, 20, 20]))
    pool.fork([4, 4, 4], [0, 1, 2], [20, 20, 20])
    shared = pool.rows[4][1]
    reserve(pool, gpu, [2, 4, 0, 1], [20] * 4, [21] * 4)
    assert pool.rows[2][1] == shared and pool.refs[shared] == 1


def test_pages_pool_that_is_too_small_changes_nothing():
    pool = qh.Pool(4, 8, 6, 16)
    gpu = pool.gpu(sb)
    reserve(pool, gpu, [0, 1], [0, 0], [48, 16])
    reserve(pool, gpu, [0, 2, 1], [40, 0, 3], [48, 70, 16])       # 5 pages wanted, 2 free; entries that want none are served
    reserve(pool, gpu, [2], [0], [32])


def test_pages_damaged_tables_are_reported():
    pool = qh.Pool(3, 4, 8, 16)
    gpu = pool.gpu(sb)
    reserve(pool, gpu, [0, 1, 2], [0, 0, 0], [64, 64, 0])
    gpu.page_table[0, 2] = 99
    gpu.held[1] = 5
    before = [t.clone() for t in (gpu.page_table, gpu.held, gpu.refs)]
    assert sb.sb_pages_release(gpu, i32([0, 1]), i32([0, 0])).cpu().tolist() == [5, 5]
    assert sb.sb_pages_fork(gpu, i32([0, 1]), i32([2, 2]), i32([64, 64])).cpu().tolist() == [5, 1]
    copies = sb.PageCopies.empty(4)
    assert sb.sb_pages_reserve(gpu, i32([0, 1]), i32([20, 0]), i32([64, 64]), copies).cpu().tolist() == [5, 5]
    assert sb.sb_pages_compact(gpu, copies).cpu().tolist() == [5] and copies.count.item() == 0
    for t, was in zip((gpu.page_table, gpu.held, gpu.refs), before):
        assert torch.equal(t, was)


def test_pages_empty_lists():
    pool = qh.Pool(3, 4, 8, 16)
    gpu = pool.gpu(sb)
    none = i32([])
    copies = sb.PageCopies.empty(2)
    copies.count.fill_(9)
    sb.sb_pages_release(gpu, none, none)
    sb.sb_pages_fork(gpu, none, none, none)
    sb.sb_pages_reserve(gpu, none, none, none, copies)
    assert copies.count.item() == 0
    pool.same(gpu)


@pytest.mark.parametrize("num,slots", [(5000, 300), (70000, 40)])
def test_pages_large_pools(num, slots):
    rng = np.random.default_rng(7)
    pool = qh.Pool(slots, 4000, num, 16)
    gpu = pool.gpu(sb)
    order = rng.permutation(slots).tolist()
    share = num // slots * 16
    reserve(pool, gpu, order, [0] * slots, [int(x) for x in rng.integers(0, share, size=slots)])
    gone = order[::3]
    assert sb.sb_pages_release(gpu, i32(gone), i32([0] * len(gone))).cpu().tolist() == pool.release(gone, [0] * len(gone))
    copies = sb.PageCopies.empty(num // 2)
    sb.sb_pages_compact(gpu, copies)
    pairs, _ = pool.compact()
    n = copies.count.item()
    assert list(zip(copies.src.tolist()[:n], copies.dst.tolist()[:n])) == pairs
    pool.same(gpu)


@pytest.mark.parametrize("layers", [1, 3])
@pytest.mark.parametrize("page_elems", [(4096,), (16400,), (3, 5)])
@pytest.mark.parametrize("dtype", [torch.uint8, torch.float32, torch.bfloat16])
def test_pages_copy_moves_whole_pages(layers, page_elems, dtype):
    if dtype == torch.uint8 and page_elems == (3, 5):
        page_elems = (3, 4)       # a page is a multiple of four bytes
    if dtype == torch.bfloat16 and page_elems == (3, 5):
        page_elems = (3, 6)
    g = torch.Generator().manual_seed(1)
    pages = 30
    lead = (layers, pages) if layers > 1 else (pages,)
    a = torch.randint(0, 100, lead + page_elems, generator=g).to(dtype).cuda()
    b = torch.randint(0, 100, lead + (7,), generator=g).float().cuda()
    want = [x.clone().view(layers, pages, -1) for x in (a, b)]
    src, dst = [3, 29, 7, 3], [0, 1, 28, 2]
    copies = sb.PageCopies(i32(src + [5, 6]), i32(dst + [8, 9]), i32([4]))    # pairs behind the count are not copied
    for w in want:
        w[:, dst] = w[:, src]
    sb.sb_pages_copy(sb.PageArrays([a, b], n_layers=layers, num_pages=pages), copies)
    assert torch.equal(a.view(layers, pages, -1), want[0]) and torch.equal(b.view(layers, pages, -1), want[1])
    copies = sb.PageCopies(i32([1, 40, 2]), i32([30, 3, 4]), i32([99]))       # ids outside the pool are skipped, the count is bounded
    sb.sb_pages_copy(sb.PageArrays([a], n_layers=layers, num_pages=pages), copies)
    want[0][:, 4] = want[0][:, 2]
    assert torch.equal(a.view(layers, pages, -1), want[0])


# ---- together -------------------------------------------------------------------------------------------------------------

def test_serving_steps_with_branches_over_an_8_bit_paged_cache():
    """A prompt is written, branched and verified step by step: pages are reserved, trees attended, accepted paths committed,
    a branch ended and the pool compacted; attention at the end equals the reference on a cache built token by token."""
    H, D, G, ps, block = 2, 64, 3, 32, 16
    rng = np.random.default_rng(40)
    slots, num = 4, 40
    pool = sb.PagePool.empty(slots, 10, num, ps)
    codes = [torch.zeros(num, ps, H, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones(num, ps // block, H, device="cuda") for _ in range(2)]
    kv = sb.QuantCache(codes[0], codes[1], scales[0], scales[1], H, D, block, page_size=ps, page_table=pool.page_table)
    arrays = sb.PageArrays(codes + scales, n_layers=1, num_pages=num)
    copies = sb.PageCopies.empty(num)
    ref = qh.Cache(rng, slots, H, D, block, 0, 200)   # a contiguous cache per slot
    hist = [0] * slots

    def rows(n):
        return [qh.bf16_of(rng.normal(size=(1, n, H, D))) for _ in range(2)]

    def reserve_all(live, grow):
        st = sb.sb_pages_reserve(pool, i32(live), i32([hist[s] for s in live]), i32([hist[s] + grow for s in live]), copies)
        assert st.cpu().tolist() == [0] * len(live)
        sb.sb_pages_copy(arrays, copies)

    # prompt of slot 0
    reserve_all([0], 75)
    k, v = rows(75)
    new, st = sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32([0, 75, 75, 75, 75]), i32(hist), max_rows=75)
    assert st.cpu().tolist() == [0] * 4
    hist = qh.append_reference(ref, k.double().numpy(), v.double().numpy(), [0, 75, 75, 75, 75], hist)
    # three branches of it
    assert sb.sb_pages_fork(pool, i32([0, 0]), i32([1, 2]), i32([75, 75])).cpu().tolist() == [0, 0]
    for s in (1, 2):
        for c in ref.codes + ref.scales:
            per = c.shape[1] // slots
            c[:, s * per:(s + 1) * per] = c[:, :per]
        hist[s] = 75
    for step in range(6):
        live = [0, 1, 2] if step < 4 else [0, 2]
        reserve_all(live, 6)
        parents = [qh.random_parents(rng, int(rng.integers(6, 30))) if s in live else [-1] for s in range(slots)]
        offs = np.concatenate([[0], np.cumsum([len(t) for t in parents])])
        k, v = rows(int(offs[-1]))
        q = qh.bf16_of(rng.normal(size=(int(offs[-1]), H * G, D)))
        check(ref, hist, parents, q, k[0], v[0], gpu=kv, window=[0, 50][step % 2], sinks=[0, 4][step % 2])
        paths = [sorted(qh.chain(t, int(rng.integers(0, len(t)))))[:6] if s in live else [] for s, t in enumerate(parents)]
        table = [p + [-1] * (6 - len(p)) for p in paths]
        accept = [len(p) - 1 for p in paths]
        # slots that are not live commit nothing: their accepted length is refused and their cache stays
        new, st = sb.sb_kv_append_quant(kv, k.cuda(), v.cuda(), i32(offs), i32(hist), max_rows=6, path_nodes=i32(table),
                                        accept_len=i32(accept), max_depth=5)
        assert [e for s, e in enumerate(st.cpu().tolist()) if s in live] == [0] * len(live)
        want = qh.append_reference(ref, k.double().numpy(), v.double().numpy(), offs, hist, paths)
        assert new.cpu().tolist() == want
        hist = want
        if step == 3:
            assert sb.sb_pages_release(pool, i32([1]), i32([0])).cpu().tolist() == [0]
            hist[1] = 0
            assert sb.sb_pages_compact(pool, copies).cpu().tolist() == [0]
            sb.sb_pages_copy(arrays, copies)
    parents = [[-1], [-1], [-1], [-1]]
    k, v = rows(4)
    q = qh.bf16_of(rng.normal(size=(4, H * G, D)))
    check(ref, hist, parents, q, k[0], v[0], gpu=kv)
