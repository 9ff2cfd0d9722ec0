"""Host side of the feed-forward operators: sizes and refusals, decided before anything is launched (no GPU)."""
import ctypes as C

import pytest

F = pytest.importorskip("paper_2110_02781_b200")
FAKE = 1 << 20                 # a 256-byte aligned address that is never dereferenced: every call below is refused on the host


def desc(rows=40, cin=64, cout=48, prec=1, act=0, stash=0, x8=0, f32=0, unaligned=0, ldx=0, ldw=0, ldy=0, ldr=0, lddx=0, lddw=0):
    return F.FfnDesc(rows, cin, cout, prec, act, stash, x8, f32, unaligned, ldx, ldw, ldy, ldr, lddx, lddw)


def size(fn, d, back):
    n = C.c_size_t()
    st = fn(C.byref(d), back, C.byref(n))
    return st, n.value


def up(n, a):
    return -(-n // a) * a


@pytest.mark.parametrize("rows,cols,parts", [(0, 5, 1), (1, 1, 1), (3, 32, 2), (7, 33, 1), (1000, 1283, 2)])
def test_image_size_follows_the_documented_layout(rows, cols, parts):
    pitch = up(cols, 32)
    assert F.ftp_checkpoint_bytes(rows, cols, parts) == parts * up(rows * (pitch + pitch // 32), 256)


def test_image_size_refusals():
    for a in ((-1, 4, 1), (1, 0, 1), (1, 4, 0), (1 << 40, 4, 1), (1, 1, 65), (1 << 37, 1 << 20, 1)):
        with pytest.raises(F.FtpError):
            F.ftp_checkpoint_bytes(*a)


def test_workspace_sizes():
    lin, gat = F.lib.ftp_linear_workspace_bytes, F.lib.ftp_gated_workspace_bytes
    assert size(lin, desc(), 0) == (0, 0) and size(gat, desc(), 0) == (0, 0)                      # bf16 read in place
    assert size(lin, desc(rows=0), 1) == (0, 0)
    assert size(lin, desc(ldx=65), 0)[1] == up(40 * 64 * 2, 256)                                   # a copy of x
    assert size(lin, desc(cout=47), 0)[1] == up(64 * 48 * 2, 256)                                 # a copy of w
    assert size(lin, desc(unaligned=1), 0)[1] == up(40 * 64 * 2, 256) + up(64 * 48 * 2, 256)
    assert size(lin, desc(prec=0), 0)[1] == up(3 * 40 * 64 * 2, 256) + up(3 * 64 * 48 * 2, 256)    # three planes of each
    assert size(lin, desc(), 1) == (0, 0)
    assert size(lin, desc(rows=300), 1)[1] == up(5 * 48 * 4, 256)                                 # sums of the bias gradient, 64 rows each
    assert size(lin, desc(act=3, stash=1), 1)[1] == up(40 * 48 * 2, 256)
    assert size(gat, desc(act=4, stash=1), 1)[1] == 2 * up(40 * 48 * 2, 256)
    assert size(gat, desc(act=4, stash=0), 1)[1] == up(2 * 40 * 48 * 2, 256) + 2 * up(40 * 48 * 2, 256)
    assert size(lin, desc(x8=1), 1)[1] == up(40 * 64 * 2, 256)
    assert size(lin, desc(rows=4, prec=0, ldx=65), 0) == (0, 0)                                   # a few tokens: read as they are
    big = size(gat, desc(rows=1 << 20, cin=8192, cout=16384, prec=0, stash=2, act=4), 1)
    assert big[0] == 0 and big[1] > 1 << 36


@pytest.mark.parametrize("kw,status", [(dict(rows=-1), 1), (dict(cin=0), 1), (dict(cout=-3), 1), (dict(prec=2), 1), (dict(act=5), 1), (dict(act=-1), 1),
                                       (dict(stash=3), 1), (dict(ldx=63), 1), (dict(ldw=47), 1), (dict(ldy=1), 1), (dict(lddx=63), 1), (dict(lddw=4), 1),
                                       (dict(rows=(1 << 31) - 1), 2), (dict(cin=1 << 30), 2), (dict(rows=1 << 30, cin=1 << 20), 2), (dict(ldx=1 << 36), 2), (dict(ldr=-1), 2)])
def test_descriptors_that_are_refused(kw, status):
    for fn in (F.lib.ftp_linear_workspace_bytes, F.lib.ftp_gated_workspace_bytes):
        assert size(fn, desc(**kw), 0)[0] == status and size(fn, desc(**kw), 1)[0] == status
    assert F.lib.ftp_linear_forward(C.byref(desc(**kw)), FAKE, FAKE, None, None, FAKE, None, None, 0, None) == status


def test_calls_that_are_refused():
    ok, L = desc(), F.lib
    ref = C.byref
    P, Q = FAKE, FAKE + 4096
    assert L.ftp_linear_forward(None, P, P, None, None, P, None, None, 0, None) == 1
    assert L.ftp_linear_forward(ref(ok), None, P, None, None, P, None, None, 0, None) == 1
    assert L.ftp_linear_forward(ref(ok), P, P, None, None, None, None, None, 0, None) == 1
    assert L.ftp_linear_forward(ref(ok), P, P, None, None, P, P, None, 0, None) == 1                      # kept values without a form
    assert L.ftp_linear_forward(ref(desc(stash=1)), P, P, None, None, P, None, None, 0, None) == 1
    assert L.ftp_linear_forward(ref(desc(stash=2)), P, P, None, None, P, P + 8, None, 0, None) == 2       # image not on 32 bytes
    assert L.ftp_linear_forward(ref(desc(x8=1)), P, P, None, None, P, None, None, 0, None) == 7
    assert L.ftp_linear_forward(ref(desc(ldr=40)), P, P, None, P, P, None, None, 0, None) == 1
    assert L.ftp_linear_forward(ref(desc(prec=0)), P, P, None, None, P, None, None, 0, None) == 3         # no workspace
    assert L.ftp_linear_forward(ref(desc(prec=0)), P, P, None, None, P, None, P, 100, None) == 3
    assert L.ftp_linear_forward(ref(desc(prec=0)), P, P, None, None, P, None, P + 16, 1 << 30, None) == 2
    assert L.ftp_linear_forward(ref(ok), P + 2, P, None, None, Q, None, None, 0, None) == 2               # not on 16 bytes, and not said so
    assert L.ftp_linear_backward(ref(desc(act=3)), P, P, None, P, None, P, P, None, P, 1 << 30, None) == 1
    assert L.ftp_linear_backward(ref(desc(stash=1)), P, P, P, P, None, P, P, None, P, 1 << 30, None) == 1
    assert L.ftp_linear_backward(ref(ok), P, P, None, None, None, P, P, None, P, 1 << 30, None) == 1
    assert L.ftp_linear_backward(ref(ok), None, P, None, P, None, None, P, None, P, 1 << 30, None) == 1   # dw without x
    assert L.ftp_linear_backward(ref(ok), P, None, None, P, None, P, None, None, P, 1 << 30, None) == 1   # dx without w
    assert L.ftp_linear_backward(ref(ok), P, P, None, P, P, None, P, None, P, 1 << 30, None) == 1         # addend without dx
    assert L.ftp_linear_backward(ref(desc(ldr=63)), P, P, None, P, P, P, P, None, P, 1 << 30, None) == 1
    assert L.ftp_linear_backward(ref(desc(x8=1)), P + 4, P, None, P, None, P, P, None, P, 1 << 30, None) == 2
    assert L.ftp_linear_forward(ref(ok), P + 1, P, None, None, Q, None, None, 0, None) == 2               # between elements
    assert L.ftp_linear_forward(ref(ok), P, P, Q + 2, None, Q, None, None, 0, None) == 2
    assert L.ftp_linear_forward(ref(desc(prec=0)), P, P, None, P + 2, Q, None, P, 1 << 30, None) == 2
    assert L.ftp_linear_backward(ref(desc(f32=1)), P, P, None, P, None, None, Q + 2, None, P, 1 << 30, None) == 2
    assert L.ftp_linear_forward(ref(ok), P, Q, None, None, P, None, None, 0, None) == 1                   # y on x, on w
    assert L.ftp_linear_forward(ref(ok), P, Q, None, None, Q, None, None, 0, None) == 1
    assert L.ftp_linear_forward(ref(desc(stash=1)), P, P, None, Q, Q, Q, None, 0, None) == 1              # kept values on y
    assert L.ftp_linear_backward(ref(ok), P, P, None, P, None, Q, Q, None, P, 1 << 30, None) == 1         # dx and dw in one place
    assert L.ftp_linear_backward(ref(ok), P, P, None, Q, None, Q, None, None, P, 1 << 30, None) == 1      # dx on dy
    assert L.ftp_checkpoint_pack(P, 4, 4, 0, 1, P, 0, None) == 1
    assert L.ftp_checkpoint_pack(P + 1, 4, 4, 0, 1, Q, 0, None) == 2
    assert L.ftp_gated_forward(ref(ok), P, P, None, P, None, None, 0, None) == 1
    assert L.ftp_gated_forward(ref(ok), P, P, P, None, None, None, 0, None) == 1
    assert L.ftp_gated_backward(ref(ok), P, P, P, None, P, None, P, P, None, P, 1 << 30, None) == 1       # one weight gradient
    assert L.ftp_gated_backward(ref(ok), None, P, P, None, P, None, P, None, None, P, 1 << 30, None) == 1 # nothing to compute the products from
    assert L.ftp_checkpoint_pack(P, 4, 4, 3, 1, P, 0, None) == 1
    assert L.ftp_checkpoint_pack(P, 4, 4, 0, 1, P + 1, 0, None) == 2
    assert L.ftp_checkpoint_pack(None, 4, 4, 0, 1, P, 0, None) == 1
    assert L.ftp_checkpoint_pack(P, 4, 4, 0, 2, P, 0, None) == 1
    assert L.ftp_checkpoint_unpack(P, -1, 4, 4, 1, P, 0, None) == 1
    assert L.ftp_checkpoint_pack(None, 0, 4, 0, 1, None, 0, None) == 0                                    # no rows: nothing to do
    assert L.ftp_linear_forward(ref(desc(rows=0)), None, None, None, None, None, None, None, 0, None) == 0


# ---- the layer kinds -----------------------------------------------------------------------------------------------
def test_layer_lists_that_are_refused():
    import synth
    L, K = synth.Layer, synth.KIND
    tail = [L(1, K["GAP"], 8, 8, 0, 1, 0, 0, 0, -1), L(1, K["FC"], 8, 3, 1, 1, 0, 0, 1, -1), L(1, K["SOFTMAX_CE"], 3, 3, 0, 1, 0, 0, 0, -1)]
    cfg = synth.config(2, 8, 1, 6, 3)
    lin = L(0, K["LINEAR"], 8, 8, 0, 1, 0, 3, 1, -1)
    F.ftp_workspace_bytes([lin] + tail, cfg)
    F.ftp_workspace_bytes([lin, lin._replace(act=0, residual_src=0)] + tail, cfg)
    F.ftp_workspace_bytes([lin, L(0, K["GATED"], 8, 8, 8, 1, 0, 4, 0, -1)] + tail, cfg)
    bad = [[lin._replace(cin=7)], [lin._replace(k=4)], [lin._replace(stride=2)], [lin._replace(pad=1)], [lin._replace(act=5)], [lin._replace(cout=0)],
           [lin, lin._replace(residual_src=1)], [lin, lin._replace(cout=8, residual_src=5)], [lin, lin._replace(kind=K["GATED"], has_bias=1)],
           [lin, lin._replace(kind=K["GATED"], has_bias=0, residual_src=0)],
           [lin._replace(cout=16), L(0, K["LINEAR"], 16, 8, 0, 1, 0, 0, 0, 0)],                       # residual of another width
           [L(0, K["ACT"], 8, 8, 0, 1, 0, 4, 0, -1)],                                                  # SILU is for the new kinds only
           [L(0, 12, 8, 8, 0, 1, 0, 0, 0, -1)]]
    for ls in bad:
        with pytest.raises(F.FtpError):
            F.ftp_workspace_bytes(ls + tail, cfg)
            pytest.fail(str(ls))


@pytest.mark.parametrize("precision", [0, 1])
def test_a_folded_batch_norm_is_no_residual_source(precision):
    """A batch norm in front of an ADD_RESIDUAL leaves the sum, not its own output: nothing may read it as a residual."""
    import synth
    L, K = synth.Layer, synth.KIND
    lin = L(0, K["LINEAR"], 8, 8, 0, 1, 0, 0, 0, -1)
    bn, add = L(0, K["BN"], 8, 8, 0, 1, 0, 0, 0, -1), L(0, K["ADD_RESIDUAL"], 8, 8, 0, 1, 0, 0, 0, 0)
    tail = [L(1, K["GAP"], 8, 8, 0, 1, 0, 0, 0, -1), L(1, K["FC"], 8, 3, 1, 1, 0, 0, 1, -1), L(1, K["SOFTMAX_CE"], 3, 3, 0, 1, 0, 0, 0, -1)]
    cfg = synth.config(2, 8, 1, 6, 3, precision=precision)
    folded = [lin, lin, bn, add]                                     # op 2 is folded into op 3
    for src in (1, 3):                                               # what is stored may be read
        F.ftp_workspace_bytes(folded + [lin._replace(residual_src=src)] + tail, cfg)
    for reader in ([lin._replace(residual_src=2)], [lin, lin._replace(residual_src=2)], [lin, bn, add._replace(residual_src=2)]):
        with pytest.raises(F.FtpError) as e:
            F.ftp_workspace_bytes(folded + reader + tail, cfg)
        assert e.value.status == 7


def test_an_addend_in_place_has_the_pitch_of_its_result():
    # residual == y and dx_addend == dx are allowed element by element: with another pitch a row would be added after it was overwritten
    ref, L, P, Q, W = C.byref, F.lib, FAKE, FAKE + 4096, FAKE + 8192
    for kw in (dict(ldr=64), dict(ldy=64), dict(ldy=64, ldr=48)):
        assert L.ftp_linear_forward(ref(desc(**kw)), P, P, None, Q, Q, None, None, 0, None) == 1, kw
    for kw in (dict(ldr=80), dict(lddx=80), dict(lddx=80, ldr=64)):
        assert L.ftp_linear_backward(ref(desc(**kw)), None, P, None, P, Q, Q, None, None, W, 1 << 30, None) == 1, kw
        assert L.ftp_gated_backward(ref(desc(stash=1, **kw)), None, P, P, P, P, Q, Q, None, None, W, 1 << 30, None) == 1, kw


def test_an_inner_classifier_is_refused_in_bf16():
    """FC computes in float: in a bf16 model only the one in front of the loss has a buffer that holds its result."""
    import synth
    L, K = synth.Layer, synth.KIND
    lin, gap = L(0, K["LINEAR"], 8, 8, 0, 1, 0, 0, 0, -1), L(0, K["GAP"], 8, 8, 0, 1, 0, 0, 0, -1)
    inner = L(0, K["FC"], 8, 8, 1, 1, 0, 0, 1, -1)
    tail = [L(0, K["FC"], 8, 3, 1, 1, 0, 0, 1, -1), L(0, K["SOFTMAX_CE"], 3, 3, 0, 1, 0, 0, 0, -1)]
    for ls in ([lin, gap, inner], [lin, gap, inner, lin], [lin, gap, lin]):
        F.ftp_workspace_bytes(ls + tail, synth.config(2, 8, 1, 6, 3))
        if inner not in ls:
            F.ftp_workspace_bytes(ls + tail, synth.config(2, 8, 1, 6, 3, precision=1))
            continue
        with pytest.raises(F.FtpError) as e:
            F.ftp_workspace_bytes(ls + tail, synth.config(2, 8, 1, 6, 3, precision=1))
        assert e.value.status == 7


@pytest.mark.parametrize("precision", [0, 1])
def test_a_residual_source_in_front_of_a_pool_is_refused_when_the_model_is_planned(precision):
    """The pool's backward pass adds no second gradient: found before a step, not in the middle of one."""
    import synth
    L, K = synth.Layer, synth.KIND
    lin, gap = L(0, K["LINEAR"], 8, 8, 0, 1, 0, 0, 0, -1), L(0, K["GAP"], 8, 8, 0, 1, 0, 0, 0, -1)
    tail = [L(0, K["FC"], 8, 3, 1, 1, 0, 0, 1, -1), L(0, K["SOFTMAX_CE"], 3, 3, 0, 1, 0, 0, 0, -1)]
    cfg = synth.config(2, 8, 1, 1, 3, precision=precision)           # one position: the pool keeps the shape
    F.ftp_workspace_bytes([lin, gap, lin._replace(residual_src=1)] + tail, cfg)
    with pytest.raises(F.FtpError) as e:
        F.ftp_workspace_bytes([lin, gap, lin._replace(residual_src=0)] + tail, cfg)
    assert e.value.status == 7
