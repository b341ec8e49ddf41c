"""The calls over 8-bit caches and pages on the GPU: what the header states beyond the ordinary cases -- the longest paths,
ranges that hold nothing, nodes, codes and scales that must not reach other results."""
import numpy as np
import pytest
import torch

import quant_helpers as qh
from paper_2605_07243_b200 import binding as sb
from test_gpu_quant import append_case, check, i32, make, same_cache, tree_of

pytestmark = pytest.mark.gpu


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
