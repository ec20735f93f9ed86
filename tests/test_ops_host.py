"""The operators beside the layer: what their entry points refuse (no GPU: every refusal comes before a launch), scratch sizes, and
the 64-bit oracle of the device tests against hand-made cases."""
import ctypes as C

import numpy as np
import pytest

import oracle.ops as ops
from paper_2510_26730_amd import binding as ef

BUF = np.zeros(1 << 16, np.uint8)
A = (BUF.ctypes.data + 255) // 256 * 256          # an aligned address that no refused call follows


@pytest.fixture(scope="module", autouse=True)
def built():
    import os
    if not os.path.exists(ef.LIB_PATH):
        from paper_2510_26730_amd import build
        build.build()
    return ef.lib()


def router(**kw):
    f = dict(n_experts=8, top_k=2, score=0, n_groups=1, groups_kept=1, group_best=1, renorm=0, scale=1.0)
    f.update(kw)
    return ef.ef_router(**f)


def refused(rc, word):
    assert rc == ef.EF_EINVAL
    assert word in ef.ef_last_error(None), ef.ef_last_error(None)


def route(r=None, logits=A, type=ef.EF_F32, ld=8, bias=None, T=4, ids=A, w=A, counts=A, offsets=A, perm=A, inv=A, work=A, bytes=1 << 15):
    r = router() if r is None else r
    return ef.lib().ef_route_scores(C.byref(r), logits, type, ld, bias, T, ids, w, counts, offsets, perm, inv, work, bytes, None)


@pytest.mark.parametrize("field,value,word", [
    ("n_experts", 0, "n_experts"), ("n_experts", 513, "n_experts"), ("top_k", 0, "top_k"), ("top_k", 9, "top_k"),
    ("score", 2, "score"), ("n_groups", 3, "n_groups"), ("n_groups", 0, "n_groups"), ("groups_kept", 2, "groups_kept"),
    ("groups_kept", 0, "groups_kept"), ("group_best", 3, "group_best"), ("group_best", 0, "group_best"), ("renorm", 2, "renorm")])
def test_router_is_checked(field, value, word):
    r = router(**{field: value})
    refused(route(r), word)
    assert ef.lib().ef_route_scores_work(C.byref(r), 4) == 0


def test_router_of_groups_is_checked():
    refused(route(router(n_groups=8, groups_kept=2, group_best=2)), "group_best")
    refused(route(router(n_groups=4, groups_kept=1, top_k=3)), "top_k")
    refused(route(router(n_experts=512, n_groups=64, groups_kept=8), ld=512), "n_groups")
    refused(route(router(n_experts=32, top_k=17), ld=32), "top_k")
    assert ef.ef_route_scores_work(4, 8, 2) > 0 and ef.ef_route_scores_work(-1, 8, 2) == 0
    assert ef.ef_route_scores_work(1 << 30, 512, 16) == 0
    # scratch for a number of tokens is enough for fewer, and small: counts of 16 tokens and their prefixes, a byte or five an expert
    for E, k, groups in ((8, 8, 1), (84, 7, 4), (200, 4, 8), (256, 8, 8), (512, 16, 1)):
        sizes = [ef.ef_route_scores_work(T, E, k, groups, groups) for T in (0, 1, 16, 17, 48, 49, 64, 65, 100, 4096, 8192, 8193, 20000, 32768, 65536, 65537, 200000)]
        assert sizes == sorted(sizes)
        assert ef.ef_route_scores_work(32768, E, k, groups, groups) <= 4096 + 16 * E * (32768 // 16)
        assert ef.ef_route_scores_work(8192, E, k, groups, groups) <= 4096 + (E + 15) // 16 * 8192


@pytest.mark.parametrize("kw,word", [
    (dict(T=-1), "T=-1"), (dict(type=ef.EF_I8), "type"), (dict(type=7), "type"), (dict(ld=7), "rows of 7"), (dict(logits=None), "null"),
    (dict(counts=None), "null"), (dict(offsets=None), "null"), (dict(work=None), "null"), (dict(work=A + 4), "misaligned"),
    (dict(ids=A + 2), "misaligned"), (dict(bias=A + 1), "misaligned"), (dict(logits=A + 2), "misaligned"),
    (dict(type=ef.EF_BF16, logits=A + 1), "misaligned"), (dict(counts=A + 1), "misaligned"), (dict(bytes=16), "scratch")])
def test_route_scores_refuses(kw, word):
    refused(route(**kw), word)


@pytest.mark.parametrize("kw,word", [
    (dict(type=ef.EF_I8), "type"), (dict(rows=-1), "rows"), (dict(K=0), "rows"), (dict(x=None), "null"), (dict(codes=None), "null"),
    (dict(scales=None), "null"), (dict(ldx=63), "overlap"), (dict(ldc=63), "overlap"), (dict(x=A + 1), "misaligned"), (dict(scales=A + 2), "misaligned")])
def test_quant_rows_refuses(kw, word):
    a = dict(x=A, type=ef.EF_BF16, ldx=64, rows=2, K=64, codes=A, ldc=64, scales=A)
    a.update(kw)
    refused(ef.lib().ef_quant_rows(a["x"], a["type"], a["ldx"], a["rows"], a["K"], a["codes"], a["ldc"], a["scales"], None), word)


def product(**kw):
    f = dict(a=A, a_scale=None, rows=None, offsets=None, w=A, w_scale=A, out=A, lda=64, ldw=64, w_group=0, ldo=32, a_type=ef.EF_BF16,
             out_type=ef.EF_F32, a_rows=4, M=4, N=32, K=64, G=1, row_div=1, swiglu=0)
    f.update(kw)
    return ef.ef_q8_product(**f)


@pytest.mark.parametrize("kw,word", [
    (dict(a=None), "null"), (dict(w=None), "null"), (dict(w_scale=None), "null"), (dict(out=None), "null"), (dict(a_type=4), "a_type"),
    (dict(out_type=ef.EF_I8), "out_type"), (dict(M=-1), "range"), (dict(N=0), "range"), (dict(K=0), "range"),
    (dict(K=131072, lda=131072, ldw=131072), "range"), (dict(a_rows=-1), "range"), (dict(G=0), "G out"), (dict(G=513), "G out"),
    (dict(swiglu=2), "swiglu"), (dict(swiglu=1, N=31), "even"), (dict(lda=63), "overlap"), (dict(ldw=48), "weight rows"),
    (dict(ldw=72), "weight rows"), (dict(w=A + 8), "weight rows"), (dict(w_group=8), "weight rows"), (dict(ldo=31), "overlap"),
    (dict(G=2), "offsets"), (dict(G=2, offsets=A, w_group=1024), "matrices overlap"), (dict(row_div=0), "row_div"),
    (dict(M=5), "product rows"), (dict(a_rows=0), "product rows"), (dict(a_type=ef.EF_I8), "a_scale"), (dict(a_scale=A), "a_scale"),
    (dict(a=A + 1), "misaligned"), (dict(out=A + 2), "misaligned"), (dict(w_scale=A + 2), "misaligned"), (dict(rows=A + 1), "misaligned"),
    (dict(offsets=A + 2), "misaligned")])
def test_matmul_q8_refuses(kw, word):
    refused(ef.lib().ef_matmul_q8(C.byref(product(**kw)), A, 1 << 15, None), word)


def test_matmul_q8_scratch():
    p = product()
    refused(ef.lib().ef_matmul_q8(C.byref(p), A, 16, None), "scratch")
    refused(ef.lib().ef_matmul_q8(C.byref(p), None, 1 << 15, None), "scratch")
    refused(ef.lib().ef_matmul_q8(C.byref(p), A + 8, 1 << 15, None), "scratch")
    assert ef.lib().ef_matmul_q8_work(C.byref(p)) >= 4 * 64 + 16
    assert ef.lib().ef_matmul_q8_work(C.byref(product(N=0))) == 0
    assert ef.lib().ef_matmul_q8(None, A, 0, None) == ef.EF_EINVAL
    assert ef.lib().ef_matmul_q8(C.byref(product(M=0)), None, 0, None) == ef.EF_OK


@pytest.mark.parametrize("kw,word", [
    (dict(y=None), "null"), (dict(w=None), "null"), (dict(out=None), "null"), (dict(y_type=ef.EF_I8), "type"), (dict(out_type=9), "type"),
    (dict(T=-1), "range"), (dict(k=0), "range"), (dict(d=0), "range"), (dict(T=1 << 30, k=2), "range"), (dict(ldy=7), "overlap"),
    (dict(ldo=7), "overlap"), (dict(y_rows=7), "rows for"), (dict(y=A + 2), "misaligned"), (dict(inv=A + 2), "misaligned")])
def test_combine_refuses(kw, word):
    a = dict(y=A, y_type=ef.EF_F32, ldy=8, y_rows=8, w=A, inv=None, T=4, k=2, d=8, out=A, out_type=ef.EF_BF16, ldo=8)
    a.update(kw)
    refused(ef.lib().ef_combine(a["y"], a["y_type"], a["ldy"], a["y_rows"], a["w"], a["inv"], a["T"], a["k"], a["d"], a["out"], a["out_type"],
                                a["ldo"], None), word)


def test_oracle_route_by_hand():
    z = np.array([[0.0, 2.0, 2.0, 1.0], [-np.inf, np.nan, -np.inf, 3.0], [-np.inf] * 4, [np.inf, 0, np.inf, 0]])
    o = ops.route_scores(z, None, 2)
    assert o["ids"].tolist() == [[1, 2], [0, 3], [0, 1], [0, 2]]
    assert o["w"][1].tolist() == [0, 1] and o["w"][2].tolist() == [0, 0] and o["w"][3].tolist() == [0.5, 0.5]
    assert o["perm"].tolist() == [2, 4, 6, 0, 5, 1, 7, 3] and o["offsets"].tolist() == [0, 3, 5, 7, 8]
    # the bias chooses, the score weighs; groups of two, one kept by the sum of its two best
    b = np.array([0.0, 0.0, 0.0, 5.0])
    o = ops.route_scores(z[:1], b, 2, sigmoid=True, n_groups=2, groups_kept=1, group_best=2, renorm=True, scale=2.0)
    assert o["ids"].tolist() == [[2, 3]]
    s = 1 / (1 + np.exp(-z[0, 2:]))
    assert np.allclose(o["w"], 2 * s / s.sum(), rtol=1e-15)


def test_oracle_quant_by_hand():
    q, s = ops.quant_rows(np.array([[127.0, 63.5, -62.5, 1.0], [0, 0, 0, 0], [1, np.inf, 0, 0], [1e-40, 0, 0, -1e-40]]))
    assert q.tolist() == [[127, 64, -62, 1], [0] * 4, [0] * 4, [0, 0, 0, 0]]
    assert s[0] == 1 and s[1] == 2.0 ** -126 and np.isnan(s[2])
    x = np.arange(-8, 8).reshape(2, 8)
    y = ops.matmul_q8(x, np.array([1.0, 0.5]), np.ones((1, 2, 8), np.int8), np.array([[1.0, 2.0]]))
    assert y.tolist() == [[-36, -72], [14, 28]]
    assert ops.combine(y, np.array([[1.0, 2.0]]), np.array([1, 0])).tolist() == [[-58, -116]]
