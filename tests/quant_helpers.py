"""Plain references of the calls over 8-bit caches and pages, in 64 bits on the CPU, and the cases that the tests make of
them.  Nothing here calls the package."""
import math

import numpy as np
import torch


# ---- e4m3 ---------------------------------------------------------------------------------------------------------------

def e4m3_table():
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        a = math.nan if (c & 127) == 127 else math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        v[c] = -a if c & 128 else a
    return v


TABLE = e4m3_table()
POSITIVE = TABLE[:127]


def e4m3_codes(x):
    """Nearest e4m3 code of every float64 (|x| <= 448), ties to the even code."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    hi = np.clip(np.searchsorted(POSITIVE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    below, above = a - POSITIVE[lo], POSITIVE[hi] - a
    code = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(a == POSITIVE[hi], hi, code)
    return (code + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def scale_of(amax):
    """Smallest power of two s >= 2^-100 with amax <= 448 s."""
    e = -100
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Cache:
    """A cache on the host: codes uint8 [layers, rows, H, D] (flat rows), scales float64 [layers, rows / block, H]."""

    def __init__(self, rng, batch, H, D, block, page_size, capacity, layers=1, spare=2, v_mag=1.0, scale_spread=1.0):
        self.batch, self.H, self.D, self.block, self.page_size, self.layers = batch, H, D, block, page_size, layers
        if page_size == 0:
            self.capacity = max(block, -(-capacity // block) * block)
            self.rows, self.table = batch * self.capacity, None
        else:
            per = max(1, -(-capacity // page_size))
            self.pages = batch * per + spare
            self.table = rng.permutation(self.pages)[:batch * per].reshape(batch, per).astype(np.int32)
            self.capacity, self.rows = per * page_size, self.pages * page_size
        self.codes, self.scales = [], []
        for mag in (1.0, v_mag):
            c = rng.integers(0, 127, size=(layers, self.rows, H, D), dtype=np.uint8)
            # magnitudes as a block scaled by its maximum has them: mostly 2^0 .. 2^8, and subnormal codes now and then
            c = np.where(rng.random(c.shape) < 0.9, 48 + c % 79, c).astype(np.uint8) | (rng.integers(0, 2, size=c.shape).astype(np.uint8) << 7)
            s = 2.0 ** (np.round(rng.normal(size=(layers, self.rows // block, H)) * scale_spread) - 8) * mag
            self.codes.append(c)
            self.scales.append(s)

    def row(self, b, j):
        if self.page_size == 0:
            return b * self.capacity + j
        return int(self.table[b, j // self.page_size]) * self.page_size + j % self.page_size

    def values(self, which, layer, b, n):
        rows = np.asarray([self.row(b, j) for j in range(n)], np.int64)
        return TABLE[self.codes[which][layer, rows]] * self.scales[which][layer, rows // self.block][:, :, None]

    def gpu(self, sb, table=None):
        """-> a QuantCache of device copies."""
        H, D, L = self.H, self.D, self.layers
        lead = (self.batch, self.capacity) if self.page_size == 0 else (self.pages, self.page_size)
        dev = [torch.from_numpy(c.reshape((L,) + lead + (H, D))).cuda() for c in self.codes]
        scl = [torch.from_numpy(s.astype(np.float32).reshape(L, lead[0], lead[1] // self.block, H)).cuda() for s in self.scales]
        t = self.table if table is None else table
        return sb.QuantCache(k_codes=dev[0], v_codes=dev[1], k_scale=scl[0], v_scale=scl[1], n_kv_heads=H, head_dim=D,
                             scale_block=self.block, page_size=self.page_size, n_layers=L,
                             page_table=None if t is None else torch.from_numpy(np.ascontiguousarray(t)).cuda())


# ---- attention ------------------------------------------------------------------------------------------------------------

def chain(parent, i):
    out = []
    while i >= 0:
        out.append(i)
        i = parent[i]
    return out


def attention_reference(cache, layer, q, k_nodes, v_nodes, P, parents, window=0, sinks=0, scale=None, q_begin=None):
    """float64 -> (out [rows, Hq, D], lse [rows, Hq], bound of |out - exact| per element, bound of the lse error).

    The bounds count, for a kernel that works as the header says: the output's rounding to bf16 (2^-8 of the value); the
    probabilities' rounding, to fp16 or bf16: at most 2^-8 of each, so 2^-8 sum p|v|; probabilities below fp16's normal
    range, off by 2^-25 of the largest product p * scale_v each; and fp32 scores and sums: a score is a sum of D products,
    off by at most D 2^-23 sum|q k|, of which a factor 2^-18 sum|q k| is kept for D <= 128 with room."""
    H, D = cache.H, cache.D
    Hq = q.shape[1]
    G = Hq // H
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, lse, tol, ltol = [], [], [], []
    node0, row0 = 0, 0
    for b, parent in enumerate(parents):
        n = len(parent)
        first = 0 if q_begin is None else q_begin[b]
        k = np.concatenate([cache.values(0, layer, b, P[b]), k_nodes[node0:node0 + n]])
        v = np.concatenate([cache.values(1, layer, b, P[b]), v_nodes[node0:node0 + n]])
        depth = [len(chain(parent, i)) - 1 for i in range(n)]
        for i in range(first, n):
            here = P[b] + depth[i]
            keys = [j for j in range(P[b]) if window == 0 or j < sinks or here - j < window]
            keys += [P[b] + a for a in sorted(chain(parent, i))
                     if window == 0 or P[b] + depth[a] < sinks or depth[i] - depth[a] < window]
            kk, vv = k[keys], v[keys]
            o_row, l_row, t_row, lt_row = [], [], [], []
            for h in range(Hq):
                qh = q[row0 + i - first, h]
                s = kk[:, h // G] @ qh * scale
                mag = np.abs(kk[:, h // G]) @ np.abs(qh) * scale
                m = s.max()
                p = np.exp(s - m)
                tot = p.sum()
                vh = vv[:, h // G]
                o_row.append(p @ vh / tot)
                l_row.append(m + math.log(tot))
                wide = p @ np.abs(vh) / tot
                ds = 2.0 ** -18 * mag.max()
                t_row.append(2.0 ** -8 * np.abs(o_row[-1]) + wide * (2.0 ** -8 + 2 * ds) + len(keys) * 2.0 ** -25 * np.abs(vh).max() / tot + 1e-30)
                lt_row.append(1e-5 * max(1.0, abs(l_row[-1])) + ds)
            out.append(o_row)
            lse.append(l_row)
            tol.append(t_row)
            ltol.append(lt_row)
        node0 += n
        row0 += n - first
    return np.asarray(out), np.asarray(lse), np.asarray(tol), np.asarray(ltol)


def random_parents(rng, n, spread=5):
    return [-1] + [int(max(0, i - 1 - int(rng.random() ** 2 * spread))) for i in range(1, n)]


def bf16_of(x):
    return torch.from_numpy(np.asarray(x, np.float32)).bfloat16()


# ---- append ---------------------------------------------------------------------------------------------------------------

def append_reference(cache, k_rows, v_rows, offsets, length, paths=None):
    """Changes `cache` as the header says; rows float64 [layers, rows, H, D]."""
    new_len = []
    for b in range(cache.batch):
        rows = list(range(offsets[b], offsets[b + 1])) if paths is None else [offsets[b] + p for p in paths[b]]
        for which, src in ((0, k_rows), (1, v_rows)):
            for layer in range(cache.layers):
                for h in range(cache.H):
                    at = 0
                    while at < len(rows):
                        t = length[b] + at
                        inside = t % cache.block
                        take = min(cache.block - inside, len(rows) - at)
                        r = cache.row(b, t)
                        blk = r // cache.block
                        x = src[layer, rows[at:at + take], h].copy()
                        bad = not np.isfinite(x).all()
                        x[~np.isfinite(x)] = 0.0
                        s = scale_of(np.abs(x).max())
                        old = cache.scales[which][layer, blk, h]
                        if inside and not math.isnan(old):
                            s = max(s, old)
                            if s != old:
                                r0 = r - inside
                                was = TABLE[cache.codes[which][layer, r0:r, h]]
                                cache.codes[which][layer, r0:r, h] = e4m3_codes(was * old / s)
                        cache.codes[which][layer, r:r + take, h] = e4m3_codes(x / s)
                        cache.scales[which][layer, blk, h] = math.nan if bad or (inside and math.isnan(old)) else s
                        at += take
        new_len.append(length[b] + len(rows))
    return new_len


# ---- pages ----------------------------------------------------------------------------------------------------------------

OK, INVALID_ARG, BOUNDS, NO_PAGES = 0, 1, 5, 7


class Pool:
    """The bookkeeping as Python lists."""

    def __init__(self, slots, max_pages, num_pages, page_size):
        self.ps, self.max_pages = page_size, max_pages
        self.rows, self.refs = [[] for _ in range(slots)], [0] * num_pages

    def pages(self, n):
        return -(-n // self.ps)

    def written(self, keep, new):
        """Logical pages that hold a position of [keep, new)."""
        return range(keep // self.ps, self.pages(new)) if new > keep else range(0)

    def _named(self, slots):
        seen, first = set(), []
        for s in slots:
            first.append(0 <= s < len(self.rows) and s not in seen)
            seen.add(s)
        return first

    def release(self, slots, keep):
        st = []
        for s, k, ok in zip(slots, keep, self._named(slots)):
            st.append(INVALID_ARG if not ok else BOUNDS if k < 0 or self.pages(k) > len(self.rows[s]) else OK)
        for s, k, e in zip(slots, keep, st):
            if e == OK:
                for page in self.rows[s][self.pages(k):]:
                    self.refs[page] -= 1
                del self.rows[s][self.pages(k):]
        return st

    def fork(self, src, dst, length):
        st = []
        for s, d, n, ok in zip(src, dst, length, self._named(dst)):
            if not ok or not 0 <= s < len(self.rows) or s == d:
                st.append(INVALID_ARG)
            else:
                st.append(BOUNDS if n < 0 or self.rows[d] or self.pages(n) > len(self.rows[s]) else OK)
        taken = [list(self.rows[s][:self.pages(n)]) if e == OK else None for s, n, e in zip(src, length, st)]
        for d, t in zip(dst, taken):
            if t is not None:
                self.rows[d] = t
                for page in t:
                    self.refs[page] += 1
        return st

    def reserve(self, slots, keep, new):
        st, wishes = [], []
        for s, k, n, ok in zip(slots, keep, new, self._named(slots)):
            if not ok:
                st.append(INVALID_ARG)
            elif k < 0 or n < k or self.pages(n) > self.max_pages or self.pages(k) > len(self.rows[s]):
                st.append(BOUNDS)
            else:
                st.append(OK)
        writers = {}
        for i, (s, k, n, e) in enumerate(zip(slots, keep, new, st)):
            if e == OK:
                for p in self.written(k, n):
                    if p < len(self.rows[s]):
                        writers.setdefault(self.rows[s][p], []).append(i)
        for i, (s, k, n, e) in enumerate(zip(slots, keep, new, st)):
            for p in self.written(k, n) if e == OK else []:
                if p >= len(self.rows[s]):
                    wishes.append((i, s, p, None))
                else:
                    page = self.rows[s][p]
                    everyone = len(writers[page]) == self.refs[page]
                    if self.refs[page] > 1 and not (everyone and writers[page][0] == i):
                        wishes.append((i, s, p, page))
        free = [p for p, r in enumerate(self.refs) if r == 0]
        if len(wishes) > len(free):
            asked = {w[0] for w in wishes}
            return [NO_PAGES if i in asked else e for i, e in enumerate(st)], []
        copies = []
        for (i, s, p, old), fresh in zip(wishes, free):
            self.refs[fresh] = 1
            if old is None:
                self.rows[s].append(fresh)
            else:
                self.refs[old] -= 1
                self.rows[s][p] = fresh
                if p * self.ps < keep[i]:
                    copies.append((old, fresh))
        return st, copies

    def compact(self):
        used = sum(r > 0 for r in self.refs)
        moving = [p for p, r in enumerate(self.refs) if r and p >= used]
        holes = [p for p, r in enumerate(self.refs) if not r and p < used]
        to = dict(zip(moving, holes))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.rows = [[to.get(p, p) for p in row] for row in self.rows]
        return sorted(to.items()), used

    def table(self):
        t = np.full((len(self.rows), self.max_pages), -1, np.int32)
        for s, row in enumerate(self.rows):
            t[s, :len(row)] = row
        return t

    def gpu(self, sb):
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
        return sb.PagePool(self.ps, torch.from_numpy(self.table()).cuda(), i32([len(r) for r in self.rows]), i32(self.refs))

    def same(self, pool):
        np.testing.assert_array_equal(pool.page_table.cpu().numpy(), self.table())
        np.testing.assert_array_equal(pool.held.cpu().numpy(), [len(r) for r in self.rows])
        np.testing.assert_array_equal(pool.refs.cpu().numpy(), self.refs)
