"""Host side of the calls over 8-bit caches and pages: refusals come before any GPU work, the binding mirrors the header,
and the tests' references hold what the header states.  No GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import quant_helpers as qh
from paper_2605_07243_b200 import binding as sb

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
A = 1 << 20   # an aligned address that is never read: every call below is refused on the host


def cache(**kw):
    s = sb._QuantCache()
    d = dict(batch=2, n_kv_heads=2, head_dim=64, scale_block=16, k_codes=A, v_codes=A, k_scale=A, v_scale=A, page_size=16,
             max_pages=4, kv_capacity=0, num_pages=8, n_layers=1, codes_layer_stride=0, scale_layer_stride=0, page_table=A)
    d.update(kw)
    for k, v in d.items():
        setattr(s, k, v)
    return s


def tree(**kw):
    s = sb._QuantTree()
    d = dict(n_q_heads=4, total_nodes=4, max_nodes=4, max_prefix=64, prefix_len=A, node_offsets=A, parent=A)
    d.update(kw)
    for k, v in d.items():
        setattr(s, k, v)
    return s


def attention(kv=None, t=None, **kw):
    kv, t = kv or cache(), t or tree()   # (held until the call returns)
    d = dict(layer=0, k=A, v=A, node_stride=0, begin=None, offsets=None, total_q=4, q=A, q_stride=0, out=A, lse=A, scale=0.0,
             window=0, sinks=0, splits=0, ws=A, ws_bytes=1 << 30, status=A)
    d.update(kw)
    return sb.load().sb_tree_attention_quant(C.addressof(kv), d["layer"], C.addressof(t), d["k"], d["v"], d["node_stride"], d["begin"],
                                             d["offsets"], d["total_q"], d["q"], d["q_stride"], d["out"], d["lse"], d["scale"], d["window"],
                                             d["sinks"], d["splits"], d["ws"], d["ws_bytes"], d["status"], None)


BAD_CACHES = [(dict(batch=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(k_codes=None), INVALID), (dict(v_scale=None), INVALID),
              (dict(k_codes=A + 8), INVALID), (dict(k_scale=A + 2), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(scale_block=8), UNSUPPORTED),
              (dict(scale_block=32), UNSUPPORTED), (dict(page_size=-16), INVALID), (dict(page_size=24), UNSUPPORTED), (dict(page_table=None), INVALID),
              (dict(max_pages=0), INVALID), (dict(num_pages=0), INVALID), (dict(page_size=0, kv_capacity=0), INVALID),
              (dict(page_size=0, kv_capacity=40), UNSUPPORTED), (dict(n_layers=0), INVALID), (dict(codes_layer_stride=8), INVALID),
              (dict(max_pages=1 << 28), UNSUPPORTED), (dict(page_size=0, kv_capacity=1 << 31), UNSUPPORTED)]


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_calls_refuse_a_bad_cache(change, code):
    kv = cache(**change)
    assert attention(kv) == code
    assert sb.load().sb_kv_append_quant(C.addressof(kv), A, A, 0, 0, A, 4, None, None, 0, 4, A, A + 64, A, None) == code
    assert sb.load().sb_tree_attention_quant_workspace_bytes(C.addressof(kv), C.addressof(tree()), 4, 0, 0, 0) == 0


@pytest.mark.parametrize("change,code", [
    (dict(prefix_len=None), INVALID), (dict(node_offsets=None), INVALID), (dict(parent=None), INVALID), (dict(n_q_heads=3), INVALID),
    (dict(n_q_heads=0), INVALID), (dict(n_q_heads=34), UNSUPPORTED), (dict(max_nodes=0), UNSUPPORTED), (dict(max_nodes=129), UNSUPPORTED),
    (dict(total_nodes=-1), INVALID), (dict(max_prefix=-1), INVALID)])
def test_attention_refuses_a_bad_tree(change, code):
    assert attention(t=tree(**change)) == code


@pytest.mark.parametrize("change,code", [
    (dict(layer=1), INVALID), (dict(layer=-1), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(q=None), INVALID),
    (dict(out=None), INVALID), (dict(status=None), INVALID), (dict(k=A + 2), INVALID), (dict(q=A + 8), INVALID), (dict(out=A + 4), INVALID),
    (dict(node_stride=64), INVALID), (dict(node_stride=132), INVALID), (dict(q_stride=128), INVALID), (dict(q_stride=260), INVALID),
    (dict(total_q=0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(window=-1), INVALID),
    (dict(window=0, sinks=4), INVALID), (dict(window=8, sinks=-1), INVALID), (dict(splits=-1), INVALID), (dict(begin=A), INVALID),
    (dict(splits=9, ws=None), WORKSPACE), (dict(splits=9, ws=A + 16), WORKSPACE), (dict(splits=9, ws_bytes=64), WORKSPACE)])
def test_attention_refuses_bad_arguments(change, code):
    t = tree(max_prefix=1 << 12) if "splits" in change else None
    kv = cache(max_pages=512) if "splits" in change else None
    assert attention(kv, t, **change) == code


def append(**kw):
    d = dict(kv=cache(), k=A, v=A, stride=0, layer=0, offsets=A, total=4, path=None, accept=None, depth=0, rows=4, len=A, new=A + 64, status=A)
    d.update(kw)
    return sb.load().sb_kv_append_quant(C.addressof(d["kv"]), d["k"], d["v"], d["stride"], d["layer"], d["offsets"], d["total"], d["path"],
                                        d["accept"], d["depth"], d["rows"], d["len"], d["new"], d["status"], None)


@pytest.mark.parametrize("change,code", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=A + 8), INVALID), (dict(offsets=None), INVALID), (dict(len=None), INVALID),
    (dict(new=None), INVALID), (dict(new=A), INVALID), (dict(status=None), INVALID), (dict(total=-1), INVALID), (dict(rows=0), INVALID),
    (dict(path=A), INVALID), (dict(accept=A), INVALID), (dict(path=A, accept=A, depth=33), UNSUPPORTED), (dict(path=A, accept=A, depth=-1), UNSUPPORTED),
    (dict(stride=64), INVALID), (dict(stride=132), INVALID), (dict(layer=-8), INVALID), (dict(layer=4), INVALID)])
def test_append_refuses_bad_arguments(change, code):
    assert append(**change) == code


def pool(**kw):
    s = sb._PagePool()
    d = dict(num_pages=8, page_size=16, n_slots=4, max_pages=4, page_table=A, held=A, refs=A)
    d.update(kw)
    for k, v in d.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("change,code", [
    (dict(num_pages=0), INVALID), (dict(n_slots=0), INVALID), (dict(max_pages=0), INVALID), (dict(page_table=None), INVALID),
    (dict(held=None), INVALID), (dict(refs=None), INVALID), (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED)])
def test_page_calls_refuse_a_bad_pool(change, code):
    lib, bad = sb.load(), pool(**change)
    p = C.addressof(bad)
    tail = (A, 1 << 20, A, None)
    assert lib.sb_pages_fork(p, 1, A, A, A, *tail) == code
    assert lib.sb_pages_reserve(p, 1, A, A, A, A, A, A, *tail) == code
    assert lib.sb_pages_release(p, 1, A, A, *tail) == code
    assert lib.sb_pages_compact(p, A, A, 4, A, A, *tail) == code
    assert lib.sb_pages_workspace_bytes(p, 1) == 0


def test_page_calls_refuse_bad_arguments():
    lib, good = sb.load(), pool()
    p = C.addressof(good)
    need = lib.sb_pages_workspace_bytes(p, 3)
    assert need > 0 and need % 256 == 0
    for ws in ((None, need), (A + 16, need), (A, need - 1)):
        assert lib.sb_pages_fork(p, 3, A, A, A, *ws, A, None) == WORKSPACE
        assert lib.sb_pages_reserve(p, 3, A, A, A, A, A, A, *ws, A, None) == WORKSPACE
        assert lib.sb_pages_release(p, 3, A, A, *ws, A, None) == WORKSPACE
    tail = (A, need, A, None)
    assert lib.sb_pages_fork(p, -1, A, A, A, *tail) == INVALID and lib.sb_pages_fork(p, 1, None, A, A, *tail) == INVALID
    assert lib.sb_pages_reserve(p, 1, A, A, None, A, A, A, *tail) == INVALID and lib.sb_pages_reserve(p, 1, A, A, A, A, A, None, *tail) == INVALID
    assert lib.sb_pages_release(p, 1, A, None, *tail) == INVALID
    assert lib.sb_pages_compact(p, A, A, 3, A, A, *tail) == INVALID      # room for fewer than num_pages / 2 pairs
    arr = (sb._PageArray * 9)()
    for a in arr:
        a.base, a.page_bytes, a.layer_stride = A, 64, 64 * 8
    r = C.addressof(arr)
    assert lib.sb_pages_copy(r, 9, 1, 8, A, A, A, 4, None) == UNSUPPORTED
    assert lib.sb_pages_copy(r, 0, 1, 8, A, A, A, 4, None) == INVALID and lib.sb_pages_copy(r, 1, 0, 8, A, A, A, 4, None) == INVALID
    assert lib.sb_pages_copy(r, 1, 1, 8, None, A, A, 4, None) == INVALID and lib.sb_pages_copy(r, 1, 1, 8, A, A, None, 4, None) == INVALID
    for change in (dict(base=None), dict(base=A + 2), dict(page_bytes=6), dict(page_bytes=0), dict(layer_stride=-4), dict(layer_stride=64)):
        one = (sb._PageArray * 1)()
        one[0].base, one[0].page_bytes, one[0].layer_stride = A, 64, 64 * 8
        for k, v in change.items():
            setattr(one[0], k, v)
        assert lib.sb_pages_copy(C.addressof(one), 1, 2, 8, A, A, A, 4, None) == INVALID, change
    assert sb.sb_status_string(7) == "too few free pages"


def test_structs_match_the_header():
    assert C.sizeof(sb._QuantCache) == 96 and sb._QuantCache.kv_capacity.offset == 56 and sb._QuantCache.page_table.offset == 88
    assert C.sizeof(sb._QuantTree) == 40 and C.sizeof(sb._PagePool) == 40 and C.sizeof(sb._PageArray) == 24


def test_binding_refuses_tensors_of_the_wrong_kind():
    codes, scales = torch.zeros(2, 32, 2, 64, dtype=torch.uint8), torch.zeros(2, 2, 2)
    ok = dict(k_codes=codes, v_codes=codes, k_scale=scales, v_scale=scales, n_kv_heads=2, head_dim=64, scale_block=16)
    kv = sb.QuantCache(**ok)
    assert kv.batch == 2 and kv.c_struct.kv_capacity == 32
    for change, err in ((dict(k_codes=codes.float()), TypeError), (dict(k_scale=scales.double()), TypeError), (dict(scale_block=24), ValueError),
                        (dict(v_scale=scales[:1]), ValueError), (dict(n_kv_heads=1), ValueError), (dict(v_codes=codes[:1]), ValueError),
                        (dict(k_codes=codes.transpose(0, 1)), ValueError), (dict(page_size=16), ValueError), (dict(n_layers=2), ValueError)):
        with pytest.raises(err):
            sb.QuantCache(**{**ok, **change})
    i32 = torch.zeros(3, dtype=torch.int32)
    t = sb.QuantTree(n_q_heads=4, prefix_len=i32[:2], node_offsets=i32, parent=i32, max_nodes=1, max_prefix=0)
    rows = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        sb.sb_tree_attention_quant(kv, t, torch.zeros(3, 4, 64, dtype=torch.bfloat16), rows, rows)
    with pytest.raises(ValueError, match="CUDA"):
        sb.sb_kv_append_quant(kv, rows, rows, i32, i32[:2], max_rows=1)
    p = sb.PagePool(16, torch.zeros(2, 4, dtype=torch.int32), i32[:2], i32)
    with pytest.raises(ValueError, match="CUDA"):
        sb.sb_pages_release(p, i32, i32)
    with pytest.raises(ValueError):
        sb.PagePool(16, torch.zeros(2, 4, dtype=torch.int32), i32, i32)
    with pytest.raises(ValueError):
        sb.PageArrays([torch.zeros(3, 5)], n_layers=2, num_pages=5)


def test_references_round_and_scale_as_the_formats_define():
    """The tests' own e4m3 rounding equals torch's cast, and their scale is the smallest that fits."""
    x = np.concatenate([np.random.default_rng(0).normal(size=4000) * 40, qh.POSITIVE, -qh.POSITIVE, (qh.POSITIVE[:-1] + qh.POSITIVE[1:]) / 2])
    x = np.clip(x, -448, 448)
    np.testing.assert_array_equal(qh.e4m3_codes(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    for a in (0.0, 1e-40, 448.0, 448.0001, 447.9, 224.0, 1.0, 3e38):
        s = qh.scale_of(a)
        assert a <= 448 * s and (s == 2.0 ** -100 or a > 448 * s / 2)


def test_page_reference_keeps_its_own_rules():
    rng = np.random.default_rng(1)
    p = qh.Pool(8, 6, 20, 16)
    for _ in range(300):
        s = [int(x) for x in rng.integers(0, 8, size=3)]
        k = rng.integers(0, 3)
        if k == 0:
            p.release(s, [int(rng.integers(0, len(p.rows[x]) * 16 + 1)) for x in s])
        elif k == 1:
            p.fork(s, [int(x) for x in rng.integers(0, 8, size=3)], [int(rng.integers(0, len(p.rows[x]) * 16 + 1)) for x in s])
        else:
            keep = [int(rng.integers(0, len(p.rows[x]) * 16 + 1)) for x in s]
            p.reserve(s, keep, [x + 20 for x in keep])
        if rng.random() < 0.2:
            p.compact()
        count = np.zeros(20, int)
        for row in p.rows:
            assert len(set(row)) == len(row) <= 6
            np.add.at(count, row, 1)
        assert count.tolist() == p.refs
