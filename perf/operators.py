"""Workloads of the 8-bit KV cache: tree attention over it, the writer of it, and the pages that hold it.

Three operators, each with its plain form in elementary torch operations (`own = False`) and through this package's
entry points (`own = True`):

  attention  sb_tree_attention_quant: draft-tree nodes (bf16 keys and values) over a committed prefix whose keys and
             values are e4m3 codes with one fp32 scale for each block of tokens and head; optional sliding window with
             first tokens that stay visible.
  append     sb_kv_append_quant: bf16 rows (a prompt, or the accepted path of a verified tree) become codes and scales.
  pages      sb_pages_release / fork / reserve / compact / copy: bookkeeping and contents of a paged cache.

A case is a dict of plain values; `prepare` makes its inputs from a seed, `run` is one call as a user makes it.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------

def _attention(**kw):
    case = dict(op="attention", batch=1, prefix_lo=2048, prefix_hi=2048, nodes_lo=1, nodes_hi=1, q_heads=32, kv_heads=8,
                head_dim=128, page_size=64, scale_block=64, window=0, sinks=0, ragged=1)
    case.update(kw)
    return case


def _append(**kw):
    case = dict(op="append", mode="prompt", batch=1, rows_lo=1, rows_hi=1, len_lo=0, len_hi=0, kv_heads=8, head_dim=128,
                page_size=64, scale_block=64, layers=1, ragged=1)
    case.update(kw)
    return case


def _pages(**kw):
    case = dict(op="pages", mode="branch", sequences=8, branches=1, len_lo=512, len_hi=4096, grow=8, layers=16, kv_heads=8,
                head_dim=128, page_size=64, scale_block=64, ragged=1)
    case.update(kw)
    return case


def listed():
    return [
        # one user, plain decoding: one new token after a 2k prefix, contiguous cache; latency is all that counts
        _attention(name="decode-one", page_size=0),
        # a serving batch, one token each, ragged prefixes on shuffled pages: the cache stream is the cost
        _attention(name="decode-batch", batch=64, prefix_lo=512, prefix_hi=8192),
        # one user, the verify forward of a 60-node draft tree
        _attention(name="verify-one", nodes_lo=60, nodes_hi=60, page_size=0),
        # a serving batch of draft trees of 32..96 nodes
        _attention(name="verify-batch", batch=16, prefix_lo=512, prefix_hi=8192, nodes_lo=32, nodes_hi=96),
        # long documents, full trees, 64 query heads
        _attention(name="verify-long", batch=4, prefix_lo=32768, prefix_hi=32768, nodes_lo=128, nodes_hi=128, q_heads=64),
        # long conversations on a layer with a 1k window and four sinks: most of the cache must not be touched
        _attention(name="verify-window", batch=16, prefix_lo=8192, prefix_hi=32768, nodes_lo=5, nodes_hi=33, window=1024,
                   sinks=4),
        # a verified step's accepted path, 1..9 tokens per sequence, all layers in one call
        _append(name="commit", mode="commit", batch=16, rows_lo=1, rows_hi=9, len_lo=512, len_hi=2048, layers=32),
        # prompts of four users, one layer
        _append(name="prompt", batch=4, rows_lo=2000, rows_hi=8192),
        # one sequence is continued twice: the smallest branch, latency counts
        _pages(name="branch-two", sequences=1, branches=1, len_lo=777, len_hi=777, layers=1),
        # sampling several continuations: eight sequences branch into eight each, sixteen layers
        _pages(name="branch-batch", sequences=8, branches=7, len_lo=512, len_hi=4096),
        # a third of 48 sequences has ended: the rest moves to the front of the pool
        _pages(name="compact", mode="compact", sequences=48, branches=0, len_lo=512, len_hi=4096),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op, ragged = rng.choice(["attention", "attention", "append", "pages"]), rng.randint(1, 1 << 20)
    head_dim = rng.choice([64, 128, 128])
    page_size = rng.choice([0, 16, 64, 64, 128])
    scale_block = rng.choice([b for b in (16, 32, 64, 128) if page_size == 0 or b <= page_size])
    if op == "attention":
        batch = _log(rng, 1, 64)
        kv_heads = rng.choice([1, 2, 4, 8])
        group = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
        nodes = _log(rng, 1, 128)
        # no more work than the largest listed case: keys * rows of the whole batch
        rows = batch * kv_heads * group * nodes
        most = max(1, min(32768, 500_000 // batch, int(1.0e9 / rows)))
        hi = _log(rng, 1, most)
        lo = rng.choice([0, hi // 4, hi])
        window, sinks = rng.choice([(0, 0), (0, 0), (_log(rng, 1, 4096), rng.choice([0, 1, 4, 130]))])
        return _attention(batch=batch, prefix_lo=lo, prefix_hi=hi, nodes_lo=rng.choice([1, max(1, nodes // 3), nodes]), nodes_hi=nodes,
                          q_heads=kv_heads * group, kv_heads=kv_heads, head_dim=head_dim, page_size=page_size,
                          scale_block=scale_block, window=window, sinks=sinks, ragged=ragged)
    if op == "append":
        kv_heads = rng.choice([1, 2, 4, 8])
        if rng.random() < 0.5:
            batch = _log(rng, 1, 64)
            return _append(mode="commit", batch=batch, rows_lo=1, rows_hi=rng.randint(1, 13), len_lo=0,
                           len_hi=_log(rng, 1, 8192 * 16 // max(16, batch)), kv_heads=kv_heads, head_dim=head_dim, page_size=page_size, scale_block=scale_block,
                           layers=_log(rng, 1, 32), ragged=ragged)
        batch = _log(rng, 1, 16)
        hi = _log(rng, 1, 32768 // batch)
        return _append(batch=batch, rows_lo=max(1, hi // 3), rows_hi=hi, len_lo=0, len_hi=rng.choice([0, 100, 1000]), kv_heads=kv_heads,
                       head_dim=head_dim, page_size=page_size, scale_block=scale_block, ragged=ragged)
    page_size = page_size or 32
    scale_block = min(scale_block, page_size)
    mode = rng.choice(["branch", "compact"])
    sequences = _log(rng, 1, 8) if mode == "branch" else _log(rng, 2, 48)
    hi = _log(rng, 1, 4096)
    return _pages(mode=mode, sequences=sequences, branches=rng.randint(1, 7) if mode == "branch" else 0, len_lo=max(1, hi // 8), len_hi=hi,
                  grow=rng.randint(1, 100), layers=_log(rng, 1, 16), kv_heads=rng.choice([1, 2, 8]), head_dim=head_dim,
                  page_size=page_size, scale_block=scale_block, ragged=ragged)


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------

class State:
    pass


def _sizes(case, seed):
    """Lengths of a case (the case's own: shapes do not change with the seed), and its trees and paths."""
    lengths, r = random.Random(case["ragged"]), random.Random(int(seed) * 7919 + 13)
    h = State()
    if case["op"] == "attention":
        h.P = [lengths.randint(case["prefix_lo"], case["prefix_hi"]) for _ in range(case["batch"])]
        h.N = [lengths.randint(case["nodes_lo"], case["nodes_hi"]) for _ in range(case["batch"])]
        # drafts branch near the root and run in chains: a parent is mostly one of the last few nodes
        h.parent = [[-1] + [max(0, i - 1 - int(r.random() ** 2 * 5)) for i in range(1, n)] for n in h.N]
        h.cap = h.P
    elif case["op"] == "append":
        h.P = [lengths.randint(case["len_lo"], case["len_hi"]) for _ in range(case["batch"])]
        h.n = [lengths.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["batch"])]
        h.cap = [p + n for p, n in zip(h.P, h.n)]
        if case["mode"] == "commit":
            h.tree = [min(128, 4 * n + 8) for n in h.n]
            h.path = [[0] + sorted(r.sample(range(1, t), n - 1)) for t, n in zip(h.tree, h.n)]
    else:
        h.P = [lengths.randint(case["len_lo"], case["len_hi"]) for _ in range(case["sequences"])]
        h.cap = h.P
        h.ended = sorted(r.sample(range(case["sequences"]), max(1, case["sequences"] // 3)))
    return h


def _pieces(n, size):
    return -(-n // size)


def _quantised(x, block):
    """x [..., tokens (a multiple of block), heads, dim] -> codes as float8_e4m3fn, scales [..., tokens/block, heads]."""
    s = x.shape
    y = x.reshape(*s[:-3], s[-3] // block, block, s[-2], s[-1])
    scale = _scale_of(y.abs().amax(dim=(-3, -1)))
    return (y / scale[..., :, None, :, None]).reshape(s).to(torch.float8_e4m3fn), scale


def _scale_of(amax):
    """The smallest power of two (at least 2^-100) that brings amax to 448 or less."""
    f, e = torch.frexp(amax)
    e = (e - 9 + (f > 0.875).int()).clamp(min=-100)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.full_like(amax, 2.0 ** -100))


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _cache(case, h, gen, layers=1):
    """Codes, scales and page table of a cache with room for h.cap tokens per sequence."""
    st = State()
    H, D, ps, sb, B = case["kv_heads"], case["head_dim"], case["page_size"], case["scale_block"], len(h.cap)
    if ps == 0:
        cap = max(sb, _pieces(max(h.cap), sb) * sb)
        rows, st.cap, st.pages, st.max_pages, st.table = B * cap, cap, 0, 0, None
    else:
        need = [_pieces(c, ps) for c in h.cap]
        st.cap, st.max_pages = 0, max(1, max(need))
        st.pages = max(1, sum(need)) + 3
        perm = torch.randperm(st.pages, generator=gen, device=DEV)[:sum(need)].to(torch.int32)
        table = torch.full((B, st.max_pages), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = perm[at:at + k]
            at += k
        st.table, rows = table, st.pages * ps
    blocks = (B, cap // sb) if ps == 0 else (st.pages, ps // sb)
    lead = (layers,) if layers > 1 else ()
    full = lead + ((B, cap, H, D) if ps == 0 else (st.pages, ps, H, D))
    st.codes, st.scales = [], []
    for which in (0, 1):
        codes = torch.empty(full, dtype=torch.uint8, device=DEV)
        scales = torch.empty(lead + blocks + (H,), dtype=torch.float32, device=DEV)
        # keys have a few large channels per head and heads of different size; values are plain
        mag = torch.exp(0.5 * torch.randn(H, 1, generator=gen, device=DEV)) * 0.7
        chan = 1.0 + 3.0 * (torch.rand(H, D, generator=gen, device=DEV) < 0.03) if which == 0 else torch.ones(H, D, device=DEV)
        flat_c, flat_s = codes.view(-1, H, D), scales.view(-1, H)
        step = max(sb, (1 << 24) // (H * D) // sb * sb)
        for r0 in range(0, layers * rows, step):
            r1 = min(layers * rows, r0 + step)
            x = torch.randn(r1 - r0, H, D, generator=gen, device=DEV) * (mag * chan)
            c, s = _quantised(x, sb)
            flat_c[r0:r1] = c.view(torch.uint8)
            flat_s[r0 // sb:r1 // sb] = s
        st.codes.append(codes)
        st.scales.append(scales)
    st.mag = mag
    return st


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 1000003 + 17)
    h = _sizes(case, seed)
    st = State()
    st.case, st.h = case, h
    H, D = case["kv_heads"], case["head_dim"]
    bf = dict(generator=gen, device=DEV)
    if case["op"] == "attention":
        st.kv = _cache(case, h, gen)
        total = sum(h.N)
        st.q = (torch.randn(total, case["q_heads"], D, **bf) * 1.5).bfloat16()
        st.k_nodes = torch.randn(total, H, D, **bf).bfloat16()
        st.v_nodes = torch.randn(total, H, D, **bf).bfloat16()
        st.prefix_len = _i32(h.P)
        st.node_offsets = _i32([0] + list(np.cumsum(h.N)))
        st.parent = _i32([p for t in h.parent for p in t])
        if own:
            from paper_2605_07243_b200 import binding as sb
            st.own_kv = _own_cache(case, st.kv)
            st.own_tree = sb.QuantTree(n_q_heads=case["q_heads"], prefix_len=st.prefix_len, node_offsets=st.node_offsets,
                                       parent=st.parent, max_nodes=max(h.N), max_prefix=max(h.P))
            need = sb.sb_tree_attention_quant_workspace_bytes(st.own_kv, st.own_tree, total, window=case["window"], sinks=case["sinks"])
            st.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
            st.out = torch.empty_like(st.q)
            st.lse = torch.empty(total, case["q_heads"], dtype=torch.float32, device=DEV)
            st.status = torch.empty(case["batch"], dtype=torch.int32, device=DEV)
    elif case["op"] == "append":
        layers = case["layers"]
        st.kv = _cache(case, h, gen, layers)
        n = h.tree if case["mode"] == "commit" else h.n
        total = sum(n)
        st.k_rows = (torch.randn(layers, total, H, D, **bf) * st.kv.mag).bfloat16()
        st.v_rows = torch.randn(layers, total, H, D, **bf).bfloat16()
        st.offsets = _i32([0] + list(np.cumsum(n)))
        st.len = _i32(h.P)
        st.max_depth = max(h.n) - 1 if case["mode"] == "commit" else 0
        st.path = st.accept = None
        if case["mode"] == "commit":
            st.path = _i32([p + [-1] * (st.max_depth + 1 - len(p)) for p in h.path])
            st.accept = _i32([len(p) - 1 for p in h.path])
        if own:
            st.own_kv = _own_cache(case, st.kv)
            st.new_len = torch.empty_like(st.len)
            st.status = torch.empty_like(st.len)
    else:
        H, ps, layers = case["kv_heads"], case["page_size"], case["layers"]
        S, K = case["sequences"], case["branches"]
        need = [_pieces(p, ps) for p in h.P]
        st.slots = S * (1 + K)
        st.max_pages = max(_pieces(p + case["grow"], ps) for p in h.P)
        st.pages = sum(need) + st.slots * (2 + _pieces(case["grow"], ps))
        table = torch.full((st.slots, st.max_pages), -1, dtype=torch.int32, device=DEV)
        perm = torch.randperm(st.pages, generator=gen, device=DEV).to(torch.int32)
        held = [0] * st.slots
        at = 0
        for i, k in enumerate(need):   # sequence i lives in slot i * (1 + K); the slots after it hold its last branches
            table[i * (1 + K), :k] = perm[at:at + k]
            held[i * (1 + K)] = k
            at += k
        for i in range(S):             # the last step's branches that are about to be dropped hold one page each
            for j in range(1, K + 1):
                table[i * (1 + K) + j, 0] = perm[at]
                held[i * (1 + K) + j] = 1
                at += 1
        refs = torch.zeros(st.pages, dtype=torch.int32, device=DEV)
        refs[perm[:at].long()] = 1
        # one buffer holds all bookkeeping, so that a step starts from a copy of it
        st.book = torch.cat([table.reshape(-1), _i32(held), refs])
        st.arrays = [torch.randint(0, 256, (layers, st.pages, ps * H * D), dtype=torch.uint8, generator=gen, device=DEV) for _ in range(2)]
        st.arrays += [torch.randint(-1 << 31, (1 << 31) - 1, (layers, st.pages, ps // case["scale_block"] * H), dtype=torch.int32,
                                    generator=gen, device=DEV) for _ in range(2)]   # the scales' bits
        if case["mode"] == "branch":
            st.losers = _i32([i * (1 + K) + j for i in range(S) for j in range(1, K + 1)])
            st.winners = _i32([i * (1 + K) for i in range(S) for j in range(1, K + 1)])
            st.fork_len = _i32([h.P[i] for i in range(S) for j in range(1, K + 1)])
            st.all = _i32(list(range(st.slots)))
            st.keep = _i32([h.P[i // (1 + K)] for i in range(st.slots)])
            st.grown = st.keep + case["grow"]
        else:
            st.losers = _i32(h.ended)
        st.zero = torch.zeros_like(st.losers)
        if own:
            from paper_2605_07243_b200 import binding as sb
            st.work_book = torch.empty_like(st.book)
            T = st.slots * st.max_pages
            st.pool = sb.PagePool(page_size=ps, page_table=st.work_book[:T].view(st.slots, st.max_pages),
                                  held=st.work_book[T:T + st.slots], refs=st.work_book[T + st.slots:])
            n = st.slots if case["mode"] == "branch" else st.pages // 2
            st.copies = sb.PageCopies.empty(n, device=DEV)
            st.layers = sb.PageArrays(st.arrays, n_layers=layers, num_pages=st.pages)
            st.workspace = torch.empty(max(256, sb.sb_pages_workspace_bytes(st.pool, st.slots)), dtype=torch.uint8, device=DEV)
            n = st.losers.numel()
            st.status = [torch.empty(k, dtype=torch.int32, device=DEV) for k in (n, n, st.slots, 1)]
    return st


def _own_cache(case, kv):
    from paper_2605_07243_b200 import binding as sb
    return sb.QuantCache(k_codes=kv.codes[0], v_codes=kv.codes[1], k_scale=kv.scales[0], v_scale=kv.scales[1],
                         n_kv_heads=case["kv_heads"], head_dim=case["head_dim"], scale_block=case["scale_block"],
                         page_size=case["page_size"], page_table=kv.table, n_layers=case.get("layers", 1))


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------

def run(state):
    op = state.case["op"]
    if own:
        return {"attention": _own_attention, "append": _own_append, "pages": _own_pages}[op](state)
    return {"attention": _plain_attention, "append": _plain_append, "pages": _plain_pages}[op](state)


def _own_attention(st):
    from paper_2605_07243_b200 import binding as sb
    out, lse, _ = sb.sb_tree_attention_quant(st.own_kv, st.own_tree, st.q, st.k_nodes, st.v_nodes, window=st.case["window"],
                                             sinks=st.case["sinks"], out=st.out, lse=st.lse, workspace=st.workspace, status=st.status)
    return out, lse


def _own_append(st):
    from paper_2605_07243_b200 import binding as sb
    new_len, _ = sb.sb_kv_append_quant(st.own_kv, st.k_rows, st.v_rows, st.offsets, st.len, max_rows=max(st.h.n), path_nodes=st.path,
                                       accept_len=st.accept, max_depth=st.max_depth, new_len=st.new_len, status=st.status)
    return _append_outputs(st, new_len)


def _own_pages(st):
    from paper_2605_07243_b200 import binding as sb
    st.work_book.copy_(st.book)
    ws = dict(workspace=st.workspace)
    sb.sb_pages_release(st.pool, st.losers, st.zero, status=st.status[0], **ws)
    if st.case["mode"] == "branch":
        sb.sb_pages_fork(st.pool, st.winners, st.losers, st.fork_len, status=st.status[1], **ws)
        sb.sb_pages_reserve(st.pool, st.all, st.keep, st.grown, st.copies, status=st.status[2], **ws)
    else:
        sb.sb_pages_compact(st.pool, st.copies, status=st.status[3], **ws)
    sb.sb_pages_copy(st.layers, st.copies)
    return (st.work_book, st.copies.src, st.copies.dst, st.copies.count) + tuple(st.arrays)


def _append_outputs(st, new_len):
    f8 = torch.float8_e4m3fn
    return (st.kv.codes[0].view(f8), st.kv.codes[1].view(f8), st.kv.scales[0], st.kv.scales[1], new_len)


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _token_rows(case, kv, b, n):
    """Row of the flat cache that holds each of the first n tokens of sequence b."""
    j = torch.arange(n, device=DEV)
    ps = case["page_size"]
    return b * kv.cap + j if ps == 0 else kv.table[b].long()[j // ps] * ps + j % ps


def _plain_attention(st):
    case, kv, h = st.case, st.kv, st.h
    H, D, G = case["kv_heads"], case["head_dim"], case["q_heads"] // case["kv_heads"]
    out, lse = torch.empty_like(st.q), torch.empty(st.q.shape[:2], dtype=torch.float32, device=DEV)
    at = 0
    for b, (P, N) in enumerate(zip(h.P, h.N)):
        rows = _token_rows(case, kv, b, P)
        keep = torch.arange(P, device=DEV)
        if case["window"]:     # a key that no node sees is not read
            keep = keep[(keep < case["sinks"]) | (P - keep < case["window"])]
            rows = rows[keep]
        kvs = []
        for which, nodes in ((0, st.k_nodes), (1, st.v_nodes)):
            codes = kv.codes[which].view(-1, H, D)[rows].view(torch.float8_e4m3fn).float()
            scale = kv.scales[which].view(-1, H)[rows // case["scale_block"]]
            kvs.append(torch.cat([codes * scale[:, :, None], nodes[at:at + N].float()]).transpose(0, 1))
        k, v = kvs
        # ancestors: a node's set is itself and its parent's
        par = st.parent[at:at + N].long()
        anc, cur = torch.eye(N, dtype=torch.bool, device=DEV), par.clone()
        depth = torch.zeros(N, dtype=torch.long, device=DEV)
        for _ in range(_tree_depth(h.parent[b])):
            live = cur >= 0
            anc |= (torch.arange(N, device=DEV)[None, :] == cur[:, None]) & live[:, None]
            depth += live
            cur = torch.where(live, par[cur.clamp(min=0)], cur)
        pos = torch.cat([keep, P + depth])
        seen = torch.cat([torch.ones(N, keep.numel(), dtype=torch.bool, device=DEV), anc], dim=1)
        if case["window"]:
            seen &= (pos[None, :] < case["sinks"]) | ((P + depth)[:, None] - pos[None, :] < case["window"])
        q = st.q[at:at + N].float().view(N, H, G, D).permute(1, 0, 2, 3).reshape(H, N * G, D)
        s = (q @ k.transpose(1, 2)) * (1.0 / math.sqrt(D))
        s = torch.where(seen.repeat_interleave(G, dim=0)[None], s, torch.full_like(s[:1, :1, :1], -math.inf))
        m = s.amax(dim=2, keepdim=True)
        p = torch.exp(s - m)
        total = p.sum(dim=2, keepdim=True)
        o = (p @ v) / total
        out[at:at + N] = o.view(H, N, G, D).permute(1, 0, 2, 3).reshape(N, H * G, D).to(out.dtype)
        lse[at:at + N] = (m + torch.log(total)).view(H, N, G).permute(1, 0, 2).reshape(N, H * G)
        at += N
    return out, lse


def _tree_depth(parent):
    d, most = [], 0
    for p in parent:
        d.append(0 if p < 0 else d[p] + 1)
        most = max(most, d[-1])
    return most


def _plain_append(st):
    case, kv, h = st.case, st.kv, st.h
    H, D, blk, layers = case["kv_heads"], case["head_dim"], case["scale_block"], case["layers"]
    offsets = np.concatenate([[0], np.cumsum(h.tree if case["mode"] == "commit" else h.n)])
    for b, (P, n) in enumerate(zip(h.P, h.n)):
        src = offsets[b] + (np.asarray(h.path[b]) if case["mode"] == "commit" else np.arange(n))
        src = torch.from_numpy(src).to(DEV)
        lo = P // blk * blk
        hi = _pieces(P + n, blk) * blk
        rows = _token_rows(case, kv, b, min(hi, kv.table.shape[1] * case["page_size"] if case["page_size"] else kv.cap))[lo:hi]
        blocks = rows[::blk] // blk
        old = (torch.arange(lo, hi, device=DEV) < P)[None, :, None, None]
        new = ((torch.arange(lo, hi, device=DEV) >= P) & (torch.arange(lo, hi, device=DEV) < P + n))[None, :, None, None]
        for which, x in ((0, st.k_rows), (1, st.v_rows)):
            codes = kv.codes[which].view(layers, -1, H, D).view(torch.float8_e4m3fn)
            scales = kv.scales[which].view(layers, -1, H)
            have = codes.view(torch.uint8)[:, rows].view(torch.float8_e4m3fn).float()
            x32 = torch.zeros_like(have)
            x32[:, P - lo:P - lo + n] = x[:, src].float()
            amax = x32.abs().view(layers, -1, blk, H, D).amax(dim=(2, 4))
            scale, before = _scale_of(amax), scales[:, blocks]
            if lo < P:
                scale[:, 0] = torch.maximum(scale[:, 0], before[:, 0])
            wide = scale.repeat_interleave(blk, dim=1)[..., None]
            was = before.repeat_interleave(blk, dim=1)[..., None]
            kept = torch.where(old, (have * was / wide).to(torch.float8_e4m3fn).float(), have)
            kept = torch.where(new, (x32 / wide).to(torch.float8_e4m3fn).float(), kept)
            codes.view(torch.uint8)[:, rows] = kept.to(torch.float8_e4m3fn).view(torch.uint8)
            scales[:, blocks] = scale
    return _append_outputs(st, st.len + _i32(h.n))


def _plain_pages(st):
    case = st.case
    ps = case["page_size"]
    book = st.book.clone()
    T = st.slots * st.max_pages
    table, held, refs = book[:T].view(st.slots, st.max_pages), book[T:T + st.slots], book[T + st.slots:]
    p = torch.arange(st.max_pages, device=DEV)

    def give_back(slots):      # every page of these slots loses one holder
        t = table[slots.long()]
        on = p[None, :] < held[slots.long()][:, None]
        refs.scatter_add_(0, torch.where(on, t, torch.zeros_like(t)).reshape(-1).long(), -on.reshape(-1).to(torch.int32))
        table[slots.long()] = -1
        held[slots.long()] = 0

    give_back(st.losers)
    if case["mode"] == "branch":
        on = p[None, :] < ((st.fork_len + ps - 1) // ps)[:, None]
        t = torch.where(on, table[st.winners.long()], torch.full_like(table[st.winners.long()], -1))
        table[st.losers.long()] = t
        held[st.losers.long()] = on.sum(dim=1).to(torch.int32)
        refs.scatter_add_(0, t.clamp(min=0).reshape(-1).long(), on.reshape(-1).to(torch.int32))
        # reserve: pages that will be written must have one holder; the last holder of a shared page keeps it when all
        # holders are in the call (the first of them in the list), every other one gets a page of its own
        first, last = (st.keep // ps)[:, None], ((st.grown + ps - 1) // ps)[:, None]
        t = table[st.all.long()]
        have = held[st.all.long()][:, None]
        writes = (p[None, :] >= first) & (p[None, :] < torch.minimum(have, last))
        ids = torch.where(writes, t, torch.zeros_like(t)).long()
        count = torch.zeros_like(refs).scatter_add_(0, ids.reshape(-1), writes.reshape(-1).to(torch.int32))
        order = torch.arange(t.shape[0], device=DEV)[:, None].expand_as(t)
        lowest = torch.full((refs.numel(),), 1 << 30, device=DEV).scatter_reduce_(
            0, ids.reshape(-1), torch.where(writes, order, torch.full_like(order, 1 << 30)).reshape(-1), "amin")
        shared = writes & (refs[ids] > 1) & ~((count[ids] == refs[ids]) & (lowest[ids] == order))
        wants = shared | ((p[None, :] >= have) & (p[None, :] < last))
        free = torch.sort((refs != 0).to(torch.int32), stable=True).indices.to(torch.int32)   # free pages first, ascending
        rank = torch.cumsum(wants.reshape(-1).to(torch.int32), 0).reshape(wants.shape) - 1
        fresh = torch.where(wants, free[rank.clamp(min=0)], t)
        copied = shared & (p[None, :] * ps < st.keep[:, None])
        refs.scatter_add_(0, ids.reshape(-1), -(shared.reshape(-1).to(torch.int32)))
        refs.scatter_add_(0, fresh.clamp(min=0).reshape(-1).long(), wants.reshape(-1).to(torch.int32))
        table[st.all.long()] = fresh
        held[st.all.long()] = torch.maximum(have, last)[:, 0].to(torch.int32)
        src, dst, count = _packed(copied.reshape(-1), t.reshape(-1), fresh.reshape(-1), st.slots)
    else:
        used = refs != 0
        n_used = used.sum()
        ids = torch.arange(refs.numel(), device=DEV)
        moving, hole = used & (ids >= n_used), ~used & (ids < n_used)
        rank = torch.cumsum(moving.to(torch.int32), 0) - 1
        holes = torch.sort((~hole).to(torch.int32), stable=True).indices
        to = torch.where(moving, holes[rank.clamp(min=0)], ids)
        table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].to(torch.int32), table))
        moved = refs.clone()
        refs.zero_()
        refs.scatter_add_(0, to, moved)
        src, dst, count = _packed(moving, ids.to(torch.int32), to.to(torch.int32), st.pages // 2)
    # contents
    real = (src >= 0).nonzero()[:, 0]
    s, d = src[real].long(), dst[real].long()
    for a in st.arrays:
        a[:, d] = a[:, s]
    return (book, src, dst, count) + tuple(st.arrays)


def _packed(mask, a, b, room):
    """The pairs (a, b) under the mask, in order, at the front of two arrays of `room` entries; -1 after them."""
    at = torch.where(mask, torch.cumsum(mask.to(torch.int32), 0) - 1, torch.full_like(mask, room, dtype=torch.int32)).long()
    outs = []
    for x in (a, b):
        y = torch.full((room + 1,), -1, dtype=torch.int32, device=DEV)
        y.scatter_(0, at, torch.where(mask, x, torch.full_like(x, -1)))
        outs.append(y[:room])
    return outs[0], outs[1], mask.sum().to(torch.int32).reshape(1)


# ---------------------------------------------------------------------------------------------------------------------
# work and 64-bit results
# ---------------------------------------------------------------------------------------------------------------------

def work(case):
    H, D, blk = case["kv_heads"], case["head_dim"], case["scale_block"]
    if case["op"] == "attention":
        P, N = (case["prefix_lo"] + case["prefix_hi"]) / 2, (case["nodes_lo"] + case["nodes_hi"]) / 2
        keys = min(P, case["window"] + min(case["sinks"], P)) if case["window"] else P
        b = keys * H * (2 * D + 8 / blk) + N * H * D * 4 + N * case["q_heads"] * (4 * D + 4)
        return {"bytes": case["batch"] * b, "flops": case["batch"] * 4.0 * N * case["q_heads"] * D * (keys + N / 2)}
    if case["op"] == "append":
        n = (case["rows_lo"] + case["rows_hi"]) / 2
        return {"bytes": case["batch"] * case["layers"] * n * H * 2 * (3 * D + 4 / blk), "flops": 0}
    ps = case["page_size"]
    page = 2 * (ps * H * D + ps // blk * H * 4) * case["layers"]
    tokens = (case["len_lo"] + case["len_hi"]) / 2
    if case["mode"] == "branch":   # the last page of each branch is copied
        moved = case["sequences"] * case["branches"]
        tables = case["sequences"] * (1 + case["branches"]) * (tokens / ps) * 8
    else:                          # the used pages that lie past the number of used pages
        had = case["sequences"] * (tokens / ps)
        used = had * 2 / 3
        pages = had + case["sequences"] * (2 + _pieces(case["grow"], ps))
        moved = used * (1 - used / pages)
        tables = pages * 16
    return {"bytes": 2 * moved * page + tables, "flops": 0}


def _e4m3_values():
    """The 256 e4m3 codes as float64: sign, four bits of exponent (bias 7), three of mantissa; 0x7f and 0xff are NaN."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        a = math.nan if (c & 127) == 127 else math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        v[c] = -a if c & 128 else a
    return torch.from_numpy(v).to(DEV)


def exact(case, seed):
    with torch.no_grad():
        if case["op"] == "attention":
            return _exact_attention(case, seed)
        if case["op"] == "append":
            return _exact_append(case, seed)
    return None


def _exact_attention(case, seed):
    st = prepare(case, seed)
    h, kv, val = st.h, st.kv, _e4m3_values()
    H, D, ps, blk = case["kv_heads"], case["head_dim"], case["page_size"], case["scale_block"]
    G = case["q_heads"] // H
    out = torch.zeros(st.q.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st.q.shape[:2], dtype=torch.float64, device=DEV)
    table = None if ps == 0 else kv.table.cpu().tolist()
    at = 0
    for b, (P, N) in enumerate(zip(h.P, h.N)):
        # the mask, node by node
        chains = []
        for i in range(N):
            c, a = [], i
            while a >= 0:
                c.append(a)
                a = h.parent[b][a]
            chains.append(c)
        seen = torch.zeros(N, P + N, dtype=torch.bool)
        for i, c in enumerate(chains):
            here = P + len(c) - 1
            if case["window"]:
                seen[i, max(0, min(P, here - case["window"] + 1)):P] = True
                seen[i, :min(P, case["sinks"])] = True
                for a in c:
                    pos = P + len(chains[a]) - 1
                    seen[i, P + a] = pos < case["sinks"] or here - pos < case["window"]
            else:
                seen[i, :P] = True
                seen[i, [P + a for a in c]] = True
        seen = seen.to(DEV)
        use = torch.nonzero(seen.any(dim=0))[:, 0]   # keys that some node sees
        for g in range(H):
            sides = []
            for codes, scales, nodes in ((kv.codes[0], kv.scales[0], st.k_nodes), (kv.codes[1], kv.scales[1], st.v_nodes)):
                if ps == 0:
                    c = codes[b, :P, g]
                    s = scales[b, :, g].double().repeat_interleave(blk)[:P]
                else:
                    ids = torch.tensor(table[b][:_pieces(P, ps)], dtype=torch.long, device=DEV)
                    c = codes[ids][:, :, g].reshape(-1, D)[:P]
                    s = scales[ids][:, :, g].double().reshape(-1).repeat_interleave(blk)[:P]
                sides.append(torch.cat([val[c.long()] * s[:, None], nodes[at:at + N, g].double()])[use])
            q = st.q[at:at + N, g * G:(g + 1) * G].double()
            score = torch.einsum("nhd,kd->nhk", q, sides[0]) / math.sqrt(D)
            score.masked_fill_(~seen[:, use][:, None, :], -math.inf)
            total = torch.logsumexp(score, dim=2)
            lse[at:at + N, g * G:(g + 1) * G] = total
            out[at:at + N, g * G:(g + 1) * G] = torch.einsum("nhk,kd->nhd", torch.exp(score - total[..., None]), sides[1])
        at += N
    return out, lse


def _exact_append(case, seed):
    """Codes and scales block by block in float64: nearest multiple of the code's own step, ties to even."""
    st = prepare(case, seed)
    h, kv, val = st.h, st.kv, _e4m3_values()
    H, D, ps, blk, layers = case["kv_heads"], case["head_dim"], case["page_size"], case["scale_block"], case["layers"]

    def nearest(x):
        step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(x / step) * step

    start = np.concatenate([[0], np.cumsum(h.tree if case["mode"] == "commit" else h.n)])
    results, scale_results = [], []
    for codes, scales, x in ((kv.codes[0], kv.scales[0], st.k_rows), (kv.codes[1], kv.scales[1], st.v_rows)):
        held = val[codes.view(layers, -1, blk, H, D).long()] if codes.numel() <= 1 << 30 else None
        if held is None:
            return None
        sc = scales.double().view(layers, -1, H)
        for b, (P, n) in enumerate(zip(h.P, h.n)):
            rows = start[b] + (np.asarray(h.path[b]) if case["mode"] == "commit" else np.arange(n))
            y = x[:, torch.from_numpy(rows).to(DEV)].double()
            t = P
            while t < P + n:
                end = min(P + n, (t // blk + 1) * blk)
                at = (b * kv.cap + t) // blk if ps == 0 else (int(kv.table[b, t // ps]) * ps + t % ps) // blk
                piece, inside = y[:, t - P:end - P], t % blk
                amax = piece.abs().amax(dim=(1, 3))
                power = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -160) / E4M3_MAX) - 1e-12).clamp(min=-100)
                s = torch.exp2(power)
                if inside:
                    s = torch.maximum(s, sc[:, at])
                    held[:, at, :inside] = nearest(held[:, at, :inside] * (sc[:, at] / s)[:, None, :, None])
                held[:, at, inside:inside + end - t] = nearest(piece / s[:, None, :, None])
                sc[:, at] = s
                t = end
        results.append(held.view(codes.shape))
        scale_results.append(sc.view(scales.shape))
    return results[0], results[1], scale_results[0], scale_results[1], None
