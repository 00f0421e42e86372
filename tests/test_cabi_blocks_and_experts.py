"""Host-side checks, without a GPU: the entry points for blocks of 128 and for experts reject bad arguments before launching anything."""
import pytest

import paper_2511_05811_amd as moss

FAKE = 0x10000  # 16-byte aligned, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def L():
    return moss.load()


def test_block_quantizers(L):
    q = lambda x=FAKE, rows=32, cols=32, ld=32, flags=3, qr=FAKE, sr=FAKE, qc=FAKE, sc=FAKE: \
        L.moss_quant_block128(x, rows, cols, ld, flags, qr, sr, qc, sc, None)
    assert q(x=None) == 1 and q(qr=None) == 1 and q(sc=None) == 1
    assert q(rows=0) == 2 and q(cols=40, ld=40) == 2 and q(rows=33) == 2 and q(ld=24) == 2
    assert q(flags=0) == 5 and q(flags=4) == 5 and q(flags=8 | 1) == 5
    assert q(x=FAKE + 2) == 3 and q(ld=36) == 3 and q(qr=FAKE + 8) == 3 and q(sr=FAKE + 2) == 3 and q(qc=FAKE + 4) == 3 and q(sc=FAKE + 1) == 3
    w = lambda x=FAKE, dt=1, rows=32, cols=32, q=FAKE, s=FAKE, qt=FAKE, st=FAKE: L.moss_quant_block128_weight(x, dt, rows, cols, q, s, qt, st, None)
    assert w(x=None) == 1 and w(q=None) == 1 and w(s=None) == 1 and w(st=None) == 1
    assert w(dt=2) == 5
    assert w(rows=0) == 2 and w(cols=48) == 2 and w(rows=40) == 2
    assert w(x=FAKE + 8) == 3 and w(q=FAKE + 4) == 3 and w(s=FAKE + 2) == 3 and w(qt=FAKE + 8) == 3 and w(st=FAKE + 1) == 3


def test_block_product(L):
    g = lambda M=16, N=16, K=32, a=FAKE, sa=FAKE, b=FAKE, sb=FAKE, block=128, out=FAKE, dt=0, ld=16, acc=0: \
        L.moss_gemm_fp8_block128(M, N, K, a, sa, b, sb, block, out, dt, ld, acc, None)
    for missing in ("a", "sa", "b", "sb", "out"):
        assert g(**{missing: None}) == 1
    assert g(M=0) == 2 and g(K=48) == 2 and g(ld=8) == 2 and g(N=-1) == 2
    assert g(block=64) == 5 and g(dt=3) == 5 and g(acc=1) == 5 and g(K=1 << 23) == 5
    assert g(a=FAKE + 8) == 3 and g(b=FAKE + 1) == 3 and g(out=FAKE + 2) == 3 and g(sa=FAKE + 2) == 3 and g(sb=FAKE + 1) == 3


def test_grouped_products(L):
    g = lambda rows=32, N=16, K=32, groups=2, off=FAKE, a=FAKE, ae=FAKE, sa=FAKE, b=FAKE, ldb=32, bs=512, sb=FAKE, sbs=1, out=FAKE, dt=0, ld=16, acc=0: \
        L.moss_gemm_fp8_mx_grouped(rows, N, K, groups, off, a, ae, sa, b, ldb, bs, sb, sbs, out, dt, ld, acc, None)
    for missing in ("off", "a", "sa", "b", "sb", "out"):
        assert g(**{missing: None}) == 1
    assert g(rows=0) == 2 and g(groups=0) == 2 and g(K=48, ldb=48) == 2 and g(ldb=16) == 2 and g(ld=8) == 2 and g(bs=-16) == 2 and g(sbs=-1) == 2
    assert g(groups=1025) == 5 and g(dt=2) == 5 and g(acc=1) == 5 and g(ldb=1 << 25) == 5
    assert g(ldb=40) == 3 and g(bs=520) == 3 and g(off=FAKE + 2) == 3 and g(a=FAKE + 8) == 3 and g(ae=FAKE + 1) == 3 and g(sb=FAKE + 2) == 3 and g(out=FAKE + 4) == 3
    d = lambda rows=64, M=16, N=16, groups=2, off=FAKE, a=FAKE, ae=FAKE, sa=FAKE, b=FAKE, be=FAKE, sb=FAKE, out=FAKE, dt=1, acc=0: \
        L.moss_gemm_fp8_mx_grouped_dw(rows, M, N, groups, off, a, ae, sa, b, be, sb, out, dt, acc, None)
    for missing in ("off", "a", "ae", "sa", "b", "be", "sb", "out"):
        assert d(**{missing: None}) == 1
    assert d(rows=48) == 2 and d(M=0) == 2 and d(groups=-1) == 2 and d(rows=0) == 2
    assert d(groups=2000) == 5 and d(dt=7) == 5 and d(dt=0, acc=1) == 5 and d(rows=1 << 25) == 5
    assert d(a=FAKE + 8) == 3 and d(be=FAKE + 2) == 3 and d(out=FAKE + 8) == 3 and d(sa=FAKE + 1) == 3


def test_expert_rows(L):
    rows = lambda *a: L.moss_expert_rows(*a)
    assert rows(64, 2, 8, 32) == (128 + 8 * 31) // 32 * 32
    assert rows(64, 2, 8, 1) == 128
    assert rows(1, 2, 64, 32) == 64                        # two experts at most have a row
    assert rows(1, 1, 1, 128) == 128
    for bad in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (1 << 31, 2, 1, 1), (-1, 1, 1, 1)):
        assert rows(*bad) == 0


@pytest.mark.parametrize("T,k,E,m", [(1, 1, 1, 1), (3, 2, 2, 32), (7, 3, 5, 32), (5, 2, 64, 128)])
def test_expert_rows_are_enough_whatever_the_routing(L, T, k, E, m):
    """The most rows that any distribution of the assignments takes, found by trying how many experts share them."""
    n = T * k
    most = max(sum(-(-c // m) * m for c in ([1] * (used - 1) + [n - used + 1])) for used in range(1, min(E, n) + 1))
    assert L.moss_expert_rows(T, k, E, m) >= most
    assert L.moss_expert_rows(T, k, E, m) % m == 0


def test_expert_calls(L):
    p = lambda e=FAKE, T=8, k=2, E=4, m=32, rows=128, ro=FAKE, src=FAKE, off=FAKE: L.moss_expert_plan(e, T, k, E, m, rows, ro, src, off, None)
    for missing in ("e", "ro", "src", "off"):
        assert p(**{missing: None}) == 1
    assert p(T=0) == 2 and p(k=0) == 2 and p(rows=0) == 2 and p(rows=96) == 2 and p(rows=130) == 2 and p(m=0) == 2
    assert p(E=1025, rows=1 << 20) == 5 and p(m=8192, rows=1 << 20) == 5
    assert p(e=FAKE + 2) == 3 and p(ro=FAKE + 1) == 3 and p(src=FAKE + 3) == 3 and p(off=FAKE + 2) == 3
    d = lambda x=FAKE, ro=FAKE, src=FAKE, T=8, k=2, rows=32, cols=64, ldx=64, ldy=64, y=FAKE, m=FAKE: \
        L.moss_expert_dispatch_bf16(x, ro, src, T, k, rows, cols, ldx, ldy, y, m, None)
    c = lambda y=FAKE, ro=FAKE, w=FAKE, T=8, k=2, rows=32, cols=64, ldy=64, ldo=64, out=FAKE: \
        L.moss_expert_combine_bf16(y, ro, w, T, k, rows, cols, ldy, ldo, out, None)
    b = lambda do=FAKE, y=FAKE, ro=FAKE, src=FAKE, w=FAKE, T=8, k=2, rows=32, cols=64, ldo=64, ldy=64, dy=FAKE, dw=FAKE, m=FAKE: \
        L.moss_expert_combine_bf16_backward(do, y, ro, src, w, T, k, rows, cols, ldo, ldy, dy, dw, m, None)
    for f, required in ((d, ("x", "ro", "src", "y", "m")), (c, ("y", "ro", "out")), (b, ("do", "y", "ro", "src", "w", "dy", "dw", "m"))):
        for missing in required:
            assert f(**{missing: None}) == 1, missing
        assert f(T=0) == 2 and f(k=0) == 2 and f(rows=0) == 2 and f(cols=60) == 2 and f(cols=72) == 2 and f(T=1 << 31) == 2
        assert f(ro=FAKE + 2) == 3
    assert d(ldx=68) == 3 and d(y=FAKE + 8) == 3 and d(m=FAKE + 1) == 3
    assert c(ldo=68) == 3 and c(out=FAKE + 8) == 3 and c(w=FAKE + 2) == 3
    assert b(ldy=68) == 3 and b(dy=FAKE + 8) == 3 and b(dw=FAKE + 2) == 3


def test_python_refuses_what_is_not_on_a_gpu():
    import torch
    x = torch.zeros((32, 64), dtype=torch.bfloat16)
    plan = dict(row_of=torch.zeros((32, 2), dtype=torch.int32), source=torch.zeros(64, dtype=torch.int32))
    for call in (lambda: moss.quant_block128(x), lambda: moss.quant_block128_weight(x), lambda: moss.expert_plan(plan["row_of"], 4),
                 lambda: moss.expert_dispatch_bf16(x, plan), lambda: moss.expert_combine_bf16(torch.zeros((64, 64), dtype=torch.bfloat16), plan)):
        with pytest.raises(AssertionError):
            call()
