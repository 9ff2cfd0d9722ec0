"""Host side of the operators around the feed-forward products: sizes and refusals, decided before anything is launched, and the
generator's known answers (no GPU)."""
import ctypes as C

import pytest

F = pytest.importorskip("paper_2110_02781_b200")
FAKE = 1 << 20                 # a 256-byte aligned address that is never dereferenced: every call below is refused on the host
P, Q, R = FAKE, FAKE + 4096, FAKE + 8192
L, ref = F.lib, C.byref


def join(rows=40, cols=64, prec=1, post=1, pre=1, eps=1e-6, alpha=1.0, beta=1.0, site=0, dropout=0.0, row0=0, gate_rows=0, **ld):
    return F.JoinDesc(rows, cols, prec, post, pre, eps, alpha, beta, site, dropout, row0, gate_rows, *(ld.get(k, 0) for k in (
        "ldu", "ldx", "lds", "ldy", "ldg", "lddu", "ldds", "lddx", "lddg")))


def fwd(d, u=P, x=P + 512, w_post=None, b_post=None, gate=None, w_pre=None, b_pre=None, rng=None, s=Q, y=R, stats=None):
    return L.ftp_join_forward(ref(d), u, x, w_post, b_post, gate, w_pre, b_pre, rng, s, y, stats, None)


def bwd(d, u=P, s=P + 512, w_post=None, b_post=None, gate=None, w_pre=None, stats=P + 1024, rng=None, dy=P + 2048, ds=P + 3584, du=Q, dx=R, dw_post=None, db_post=None,
        dw_pre=None, db_pre=None, dgate=None, ws=None, nws=0):
    return L.ftp_join_backward(ref(d), u, s, w_post, b_post, gate, w_pre, stats, rng, dy, ds, du, dx, dw_post, db_post, dw_pre, db_pre, dgate, ws, nws, None)


@pytest.mark.parametrize("kw,status", [(dict(rows=-1), 1), (dict(cols=0), 1), (dict(cols=16385), 7), (dict(prec=2), 1), (dict(post=3), 1), (dict(pre=-1), 1), (dict(eps=-1.0), 1),
                                       (dict(eps=float("nan")), 1), (dict(alpha=float("inf")), 1), (dict(beta=float("nan")), 1), (dict(dropout=-0.1), 1),
                                       (dict(dropout=1.5), 1), (dict(dropout=float("nan")), 1), (dict(dropout=0.5, site=1 << 24), 2), (dict(dropout=0.5, site=-1), 2),
                                       (dict(dropout=0.5, row0=-1), 2), (dict(dropout=0.5, row0=1 << 37), 2), (dict(gate_rows=-1), 1), (dict(rows=1 << 31), 2),
                                       (dict(ldu=63), 1), (dict(ldx=8), 1), (dict(lds=63), 1), (dict(ldy=-1), 1), (dict(lddg=1), 1), (dict(lddx=1 << 36), 2)])
def test_join_descriptors_that_are_refused(kw, status):
    d, n = join(**kw), C.c_size_t()
    assert L.ftp_join_workspace_bytes(ref(d), ref(n)) == status
    assert fwd(d, rng=P) == status and bwd(d, rng=P, ws=P, nws=1 << 40) == status


def test_join_calls_that_are_refused():
    ok = join()
    assert L.ftp_join_forward(None, *([P] * 11), None) == 1 and L.ftp_join_workspace_bytes(ref(ok), None) == 1
    assert fwd(ok, u=None, x=None) == 1 and fwd(ok, y=None) == 1 and fwd(ok, s=None) == 1
    assert fwd(join(pre=0)) == 1                                                      # y without its norm
    assert fwd(ok, u=None, s=None) == 1 and fwd(join(post=0, alpha=2.0), u=None, s=None) == 1
    assert fwd(join(post=0, dropout=0.5), u=None, s=None, rng=P) == 1 and fwd(join(post=0), u=None, s=None, gate=P) == 1
    assert fwd(join(post=0), w_post=P) == 1 and fwd(join(pre=0), y=None, b_pre=P) == 1
    assert fwd(join(gate_rows=3)) == 1                                                # rows of no gate
    assert fwd(join(dropout=0.5)) == 1 and fwd(join(dropout=0.5), rng=P + 4) == 2     # no words, words between words
    assert fwd(ok, u=P + 1) == 2 and fwd(ok, w_pre=P + 2) == 2 and fwd(ok, gate=P + 2) == 2 and fwd(ok, stats=P + 6) == 2
    assert fwd(ok, s=P) == 1 and fwd(ok, y=P + 512) == 1 and fwd(ok, y=Q) == 1 and fwd(ok, w_pre=Q) == 1 and fwd(ok, stats=R) == 1
    assert fwd(join(lds=80), s=P + 512) == 1                                          # the sum in place of x with another pitch
    assert fwd(join(rows=0), u=None, x=None, s=None, y=None) == 0
    n = C.c_size_t()
    assert L.ftp_join_workspace_bytes(ref(join(rows=0)), ref(n)) == 0 and n.value == 0
    assert L.ftp_join_workspace_bytes(ref(join(rows=5000)), ref(n)) == 0 and n.value > 0
    big = dict(ws=P, nws=1 << 30)
    assert bwd(ok, dy=None, **big) == 1 and bwd(join(pre=0), dy=None, ds=None, **big) == 1 and bwd(ok, s=None, **big) == 1 and bwd(ok, u=None, **big) == 1
    assert bwd(ok, stats=None, **big) == 1 and bwd(join(pre=0), **big) == 1           # dy of a norm that is not there
    assert bwd(join(post=0), dw_post=P + 256, **big) == 1 and bwd(join(pre=0), dy=None, dw_pre=P + 256, **big) == 1
    assert bwd(ok, dgate=P + 256, **big) == 1 and bwd(join(gate_rows=2), **big) == 1
    assert bwd(ok, du=P, **big) == 1 and bwd(ok, dx=P + 2048, **big) == 1 and bwd(ok, du=R, **big) == 1 and bwd(ok, du=P + 3584, **big) == 1
    assert bwd(join(lddx=80), dx=P + 3584, **big) == 1                                # dx in place of ds with another pitch
    assert bwd(ok, dw_post=Q + 2, **big) == 2 and bwd(ok, ds=P + 3, **big) == 2
    assert bwd(join(rows=5000)) == 3 and bwd(join(rows=5000), ws=P, nws=64) == 3 and bwd(join(rows=5000), ws=P + 16, nws=1 << 30) == 2
    assert bwd(join(rows=0), u=None, s=None, stats=None, dy=None, ds=None, du=None, dx=None) == 0


def test_dropout_calls_that_are_refused():
    drop = lambda x=P, y=Q, rows=4, cols=8, ldx=0, ldy=0, prec=1, p=0.5, rng=R, site=0, row0=0: L.ftp_dropout(  # noqa: E731
        x, y, rows, cols, ldx, ldy, prec, p, rng, site, row0, None)
    assert drop(prec=3) == 1 and drop(rows=-1) == 1 and drop(cols=0) == 1 and drop(ldx=7) == 1 and drop(ldy=7) == 1 and drop(p=1.01) == 1 and drop(p=-1.0) == 1
    assert drop(x=None) == 1 and drop(y=None) == 1 and drop(rng=None) == 1 and drop(rng=R + 4) == 2 and drop(x=P + 1) == 2 and drop(y=R) == 1
    assert drop(x=Q, ldx=16) == 1 and drop(rows=1 << 38) == 2 and drop(cols=1 << 30) == 2 and drop(site=1 << 24) == 2 and drop(row0=-1) == 2 and drop(row0=1 << 39) == 2
    assert drop(rows=0, x=None, y=None) == 0


def rec(seqs=2, n=40, rows=0, cols=64, prec=1, act=4, coupled=1, **ld):
    return F.RecurrenceDesc(seqs, n, rows, cols, prec, act, coupled, *(ld.get(k, 0) for k in ("ldf", "ldv", "ldo", "ldy", "lddf", "lddv", "lddo")))


def test_recurrence_calls_that_are_refused():
    def f(d=None, f=P, v=P + 256, o=P + 512, h0=None, off=None, y=Q, h1=None, st=None, **kw):
        return L.ftp_recurrence_forward(ref(d or rec(**kw)), f, v, o, h0, off, y, h1, st, None)

    def b(f=P, v=P + 256, o=P + 512, st=P + 768, off=None, dy=P + 1024, dh1=None, df=Q, dv=Q + 256, do=Q + 512, dh0=None, **kw):
        return L.ftp_recurrence_backward(ref(rec(**kw)), f, v, o, st, off, dy, dh1, df, dv, do, dh0, None)
    for call in (f, b):
        assert call(seqs=-1) == 1 and call(n=-1) == 1 and call(cols=0) == 1 and call(prec=2) == 1 and call(act=5) == 1 and call(rows=-1) == 1
        assert call(rows=81) == 1 and call(rows=80, off=None, seqs=0) in (0, 1)        # rows that are not seqs x len
        assert call(n=1 << 31) == 2 and call(seqs=1 << 31) == 2 and call(cols=1 << 30) == 2 and call(seqs=1 << 20, n=1 << 20) == 2
        assert call(ldf=63) == 1 and call(ldv=1) == 1 and call(ldo=63) == 1 and call(ldy=63) == 1 and call(ldf=1 << 36) == 2
        assert call(rows=1 << 31, off=R, cols=1) == 2 and call(rows=80, off=R + 2) == 2
        assert call(f=None) == 1 and call(v=None) == 1 and call(f=P + 1) == 2 and call(o=None, act=4) == 1
    assert f(y=None) == 1 and f(y=P) == 1 and f(y=Q, h1=Q) == 1 and f(h0=Q) == 1 and f(st=P) == 1 and f(h1=Q + 6) == 2
    assert f(seqs=0) == 0
    assert b(dy=None) == 1 and b(st=None) == 1 and b(df=None) == 1 and b(dv=None) == 1 and b(do=None) == 1 and b(o=None, act=0) == 1 and b(lddv=63) == 1
    assert b(df=P) == 1 and b(dv=P + 1024) == 1 and b(df=Q + 256) == 1 and b(dh1=Q) == 1 and b(dh0=P + 768) == 1 and b(dh0=P + 2) == 2
    assert b(seqs=0) == 0
    n = C.c_int64()
    assert L.ftp_recurrence_states(ref(rec()), None) == 1 and L.ftp_recurrence_states(ref(rec()), ref(n)) == 0 and n.value == 80 // 16 + 2
    assert F.ftp_recurrence_states(100, 3) == 9


def test_recurrence_rows_that_are_not_those_of_its_sequences_are_refused():
    for seqs, n, rows, status in ((0, 40, 80, 1), (2, 40, 81, 1), (2, 0, 80, 1), (0, 40, 0, 0)):
        d = rec(seqs=seqs, n=n, rows=rows)
        assert L.ftp_recurrence_forward(ref(d), P, P + 256, P + 512, None, None, Q, None, None, None) == status
        assert L.ftp_recurrence_backward(ref(d), P, P + 256, P + 512, P + 768, None, P + 1024, None, Q, Q + 256, Q + 512, None, None) == status


def test_logprob_calls_that_are_refused():
    def f(x=P, rows=4, vocab=64, ld=0, prec=1, scale=1.0, t=P + 2048, logp=Q, ent=None, lse=None, top=None, tl=None, k=0):
        return L.ftp_logprob_forward(x, rows, vocab, ld, prec, scale, t, logp, ent, lse, top, tl, k, None)

    def b(x=P, rows=4, vocab=64, ld=0, prec=1, scale=1.0, t=P + 2048, lse=P + 1024, ent=None, dl=P + 1536, dh=None, dx=Q, ldd=0):
        return L.ftp_logprob_backward(x, rows, vocab, ld, prec, scale, t, lse, ent, dl, dh, dx, ldd, None)
    for call in (f, b):
        assert call(prec=2) == 1 and call(rows=-1) == 1 and call(vocab=0) == 1 and call(ld=63) == 1 and call(scale=0.0) == 1 and call(scale=-1.0) == 1
        assert call(scale=float("inf")) == 1 and call(scale=2e18) == 1 and call(scale=float("nan")) == 1 and call(x=None) == 1 and call(x=P + 1) == 2 and call(t=P + 2) == 2 and call(t=None) == 1
        assert call(rows=1 << 28) == 2 and call(vocab=1 << 30) == 2 and call(ld=1 << 36) == 2 and call(rows=0, x=None) == 0
    assert f(k=33, top=R) == 1 and f(k=-1) == 1 and f(k=5) == 1 and f(top=R) == 1 and f(tl=R) == 1 and f(vocab=4, k=5, top=R) == 1
    assert f(logp=P) == 1 and f(ent=Q) == 1 and f(k=2, top=Q) == 1 and f(lse=Q + 2) == 2
    assert b(lse=None) == 1 and b(dx=None) == 1 and b(dl=None) == 1 and b(dh=R) == 1 and b(dx=P, ldd=80) == 1 and b(dx=P + 1024) == 1 and b(ldd=63) == 1 and b(dx=Q + 1) == 2


def test_generator_known_answers():
    """The published vectors of Philox 4x32-10, and the vectorised form against the plain one."""
    from token_helpers import keep_mask, philox
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    key, step, site, row0, cols, p = (5 << 40) + 77, (9 << 33) + 3, 12, 1 << 34, 19, 0.3
    got, factor = keep_mask(3, cols, p, key, step, site, row0)
    cut = 19661
    assert factor == 65536 / (65536 - cut)
    for r in range(3):
        for c in range(cols):
            n = (row0 + r) * 3 + c // 8
            w = philox((n & 0xFFFFFFFF, n >> 32 | site << 8, step & 0xFFFFFFFF, step >> 32), (key & 0xFFFFFFFF, key >> 32))[c % 8 // 2]
            assert bool(got[r, c]) == ((w >> 16 if c % 2 else w & 0xFFFF) >= cut)
