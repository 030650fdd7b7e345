"""The plan of the transposed mask (SPLAT_PLAN_GRAD): every non-zero of the
oracle's mask in exactly one tile under its key's mask, tiles of a group
disjoint, the states and the rows with a single key as the masks say.  CPU only.
"""
import ctypes

import numpy as np
import pytest
from hypothesis import given, settings, strategies as st

import paper_2407_16847_amd as splat
from oracle import masks as om

CASES = [
    ("window", {"w": 0}, 70), ("window", {"w": 5}, 1), ("window", {"w": 40}, 700),
    ("blocked", {"block": 33}, 300), ("strided_local", {"local": 40, "stride": 33}, 500),
    ("strided_local", {"local": 128, "stride": 128}, 1100), ("dilated", {"w": 33, "dilation": 3}, 400),
    ("dilated", {"w": 8, "dilation": 4}, 3), ("window_global", {"w": 3, "n_global": 70}, 900),
    ("full", {}, 128), ("full", {}, 333),
]


def _dense(a):
    """The mask that the transposed plan describes, checked on the way."""
    g, keys, tiles, masks, lone = a.export_grad_plan()
    L = a.L
    M = np.zeros((L, L), dtype=np.int64)
    assert sorted(keys.tolist()) == list(range(L))
    assert g[:, 1].sum() == L and (g[:, 1] > 0).all() and (g[:, 1] <= 128).all()
    order = [int(e - b) for _, _, b, e in g]
    assert order == sorted(order, reverse=True)
    rp, _ = a.export()
    single = np.diff(rp) == 1
    for off, n, t0, t1 in g:
        seen = np.zeros(L, dtype=bool)
        for t in range(t0, t1):
            qb, qs, nq, flags, block = (int(x) for x in tiles[t])
            q = qb + qs * np.arange(nq)
            assert 1 <= nq <= 64 and qs >= 1 and q[-1] < L and not seen[q].any()
            seen[q] = True
            assert int(lone[t]) == sum(1 << int(u) for u in np.nonzero(single[q])[0])
            partial = False
            for w in range(4):
                state = (flags >> (8 + 2 * w)) & 3
                ks = keys[off + 32 * w: off + min(n, 32 * w + 32)]
                partial |= state == 1
                if state == 3:
                    assert nq == 64 and len(ks) and not single[q].any()
                    M[np.ix_(q, ks)] += 1
                    if block >= 0:
                        assert (masks[block, 32 * w: 32 * w + len(ks)] == ~np.uint64(0)).all()
                    continue
                bits = masks[block, 32 * w: 32 * w + 32] if block >= 0 else np.zeros(32, np.uint64)
                if state == 0:
                    assert not bits.any()
                assert not bits[len(ks):].any()
                for m, j in enumerate(ks):
                    for u in range(64):
                        if (int(bits[m]) >> u) & 1:
                            assert u < nq
                            M[q[u], j] += 1
            assert (block >= 0) == partial
    return M


@pytest.mark.parametrize("kind,params,L", CASES)
def test_grad_plan_covers_the_mask(kind, params, L):
    a = splat.Acsr(splat.Pattern.named(kind, params, L), grad=True)
    assert a.info()["grad"] == 1
    assert np.array_equal(_dense(a), om.dense_mask(kind, params, L).astype(np.int64))


def test_grad_plan_of_empty_and_partial_masks():
    a = splat.Acsr(splat.Pattern.from_terms(100, []), grad=True)
    assert not _dense(a).any()
    M = np.zeros((150, 150), dtype=np.uint8)
    M[10:90, 20:30] = 1
    M[100, 0::7] = 1
    M[149, 149] = 1
    assert np.array_equal(_dense(splat.Acsr(mask=M, grad=True)), M)


@settings(max_examples=60, deadline=None)
@given(st.integers(1, 200).flatmap(lambda L: st.tuples(st.just(L), st.lists(
    st.tuples(st.integers(0, L - 1), st.integers(1, 9), st.integers(0, 40)), min_size=L, max_size=L))))
def test_grad_plan_of_random_masks(case):
    L, rows = case
    M = np.zeros((L, L), dtype=np.uint8)
    for i, (start, stride, count) in enumerate(rows):
        M[i, start: min(L, start + stride * count): stride] = 1
    assert np.array_equal(_dense(splat.Acsr(mask=M, grad=True)), M)


def test_global_columns_have_groups_of_their_own():
    """Columns that every row has do not make the other keys of a group walk
    every row: the rows that the groups walk stay near those that they need."""
    a = splat.Acsr(splat.Pattern.strided_local(2048, 128, 128), grad=True)
    g, keys, tiles, _, _ = a.export_grad_plan()
    assert set(keys[g[0, 0]: g[0, 0] + g[0, 1]]) >= set(range(127, 1024, 128))
    assert len(tiles) <= 32 + 18 * 5


def test_refusals():
    a = splat.Acsr(splat.Pattern.window(64, 4))
    assert a.info()["grad"] == 0
    with pytest.raises(splat.SplatError, match="SPLAT_PLAN_GRAD"):
        a.export_grad_plan()
    lib, h = splat.load(), ctypes.c_void_p()
    m = np.ones((8, 8), dtype=np.uint8)
    at = m.ctypes.data_as(ctypes.c_void_p)
    for flags in (1, 2, 4, 9, 16):
        assert lib.splat_acsr_from_mask_ex(8, at, flags, ctypes.byref(h)) == 1
    assert lib.splat_acsr_from_mask_ex(8, at, 8, None) == 1
    with pytest.raises(ValueError):
        splat.Acsr(mask=m, columns=True, grad=True)


def test_with_other_flags():
    """The transposed plan does not depend on the plan's other options."""
    pat = splat.Pattern.window(300, 20)
    ref = splat.Acsr(pat, grad=True).export_grad_plan()
    for kw in (dict(columns=True), dict(span=False), dict(columns=True, span=False)):
        got = splat.Acsr(pat, grad=True, **kw).export_grad_plan()
        assert all(np.array_equal(x, y) for x, y in zip(ref, got))


def test_sanitized(tmp_path):
    """The planner built with the address and undefined-behaviour sanitizers, with
    the transposed plan asked for, over the cases above and random masks."""
    import test_host_sanitized as sanitized
    import os
    import shutil
    import subprocess
    cxx = shutil.which(os.environ.get("CXX", "g++"))
    exe = str(tmp_path / "host_check")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
                        "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-I" + os.path.join(sanitized.ROOT, "include"), *sanitized.SRC, "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    pats = [splat.Pattern.named(k, p, L) for k, p, L in CASES] + [splat.Pattern.from_terms(100, [])]
    out = sanitized.run(exe, [sanitized.desc_line(p, splat.PLAN_GRAD) for p in pats])
    assert all(x["status"] == 0 for x in out)
