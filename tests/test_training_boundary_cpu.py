"""Host-only checks of the entry points for dropout, layer norm and losses over many classes: arguments are refused before the device is
touched, and workspace queries follow the shapes."""
from paper_1810_09868_amd import binding as B

A = 4096  # a 16-byte aligned address that is never used
NAN = float("nan")


def test_dropout_is_refused_on_the_host():
    L = B.lib()
    call = lambda dt=0, N=2, C=10, ldx=10, x=A, p=0.5, r=A, layer=1, y=2 * A, ldy=10: L.vgg_dropout(dt, N, C, ldx, x, p, r, layer, y, ldy, None)  # noqa: E731
    assert call(x=None) == call(y=None) == call(r=None) == -1
    assert call(dt=2) == -3
    assert call(N=0) == call(C=0) == call(ldx=9) == call(ldy=9) == call(y=A, ldy=11) == call(p=-0.1) == call(p=1.5) == call(p=NAN) == call(layer=65536) == -2
    assert call(N=(1 << 23) + 1) == call(C=(1 << 30) + 1, ldx=1 << 31, ldy=1 << 31) == -2
    assert call(x=A + 2) == call(y=A + 4) == call(r=A + 8) == -4


def test_layer_norm_is_refused_on_the_host():
    L = B.lib()
    call = lambda dt=1, N=2, C=10, ldx=10, x=A, g=A, b=A, eps=1e-5, p=0.5, r=A, layer=1, y=2 * A, ldy=10, st=A: L.vgg_layer_norm(  # noqa: E731
        dt, N, C, ldx, x, g, b, eps, p, r, layer, y, ldy, st, None)
    assert call(x=None) == call(y=None) == call(r=None) == -1 and call(dt=-1) == -3
    assert call(N=0) == call(C=-1) == call(ldx=9) == call(ldy=9) == call(y=A, ldy=12) == call(eps=-1.0) == call(eps=NAN) == call(p=2.0) == call(layer=1 << 16) == -2
    assert call(g=A + 4) == call(b=A + 4) == call(st=A + 4) == call(r=A + 8) == -4
    back = lambda dt=1, gt=1, N=2, C=10, ldx=10, x=A, g=A, st=A, p=0.5, r=A, layer=1, lddy=10, dy=2 * A, dx=3 * A, lddx=10, dg=A, db=A, ws=A, nb=1 << 40: (  # noqa: E731
        L.vgg_layer_norm_bwd(dt, gt, N, C, ldx, x, g, st, p, r, layer, lddy, dy, dx, lddx, dg, db, 1, ws, nb, None))
    assert back(x=None) == back(st=None) == back(dy=None) == back(dx=None) == back(r=None) == -1
    assert back(dt=2) == back(gt=2) == back(dt=0, gt=1) == -3
    assert back(N=0) == back(ldx=9) == back(lddy=9) == back(lddx=9) == back(dx=2 * A, lddx=11) == back(dx=A, lddx=11) == back(dx=A, gt=0) == back(p=NAN) == -2
    assert back(dy=2 * A + 2) == back(dg=A + 4) == back(ws=A + 4) == -4
    need = B.vgg_layer_norm_bwd_workspace_bytes(B.BF16, B.BF16, 1000, 4096)
    assert need > 0 and back(N=1000, C=4096, ldx=4096, lddy=4096, lddx=4096, nb=need - 1) == back(N=1000, C=4096, ldx=4096, lddy=4096, lddx=4096, ws=None) == -5
    assert B.vgg_layer_norm_bwd_workspace_bytes(B.F32, B.BF16, 100, 4096) == B.vgg_layer_norm_bwd_workspace_bytes(9, 9, 100, 4096) == 0
    assert B.vgg_layer_norm_bwd_workspace_bytes(B.F32, B.F32, 0, 4096) == 0


def test_losses_over_classes_are_refused_on_the_host():
    L = B.lib()
    call = lambda dt=0, N=2, i=8, k=10, a=A, w=A, b=A, y=A, lo=A, st=A, ws=A, nb=1 << 50: L.vgg_fc_xent(dt, N, i, k, a, w, b, y, lo, st, ws, nb, None)  # noqa: E731
    assert call(a=None) == call(w=None) == call(y=None) == call(lo=None) == -1 and call(dt=2) == -3
    assert call(N=0) == call(i=0) == call(k=0) == call(N=(1 << 22) + 1) == call(i=(1 << 20) + 1) == call(k=(1 << 24) + 1) == -2
    assert call(a=A + 2) == call(w=A + 8) == call(b=A + 4) == call(y=A + 2) == call(lo=A + 4) == call(st=A + 8) == call(ws=A + 8) == -4
    assert call(ws=None) == call(nb=B.vgg_fc_xent_workspace_bytes(B.F32, 2, 8, 10) - 1) == -5
    assert call(y=A + 4, nb=0) == -5                # a part of a longer sequence of labels is taken
    back = lambda dt=1, gt=1, N=2, i=8, k=10, a=A, w=A, b=A, y=A, st=A, g=A, da=A, dw=A, db=A, ws=A, nb=1 << 50: (  # noqa: E731
        L.vgg_fc_xent_bwd(dt, gt, N, i, k, a, w, b, y, st, g, da, dw, db, 1, ws, nb, None))
    assert back(a=None) == back(w=None) == back(y=None) == back(st=None) == back(g=None) == back(da=None, dw=None, db=None) == -1
    assert back(dt=3) == back(dt=0, gt=1) == back(gt=5) == -3 and back(N=-1) == back(i=0) == back(k=0) == -2
    assert back(da=A + 2) == back(dw=A + 2) == back(db=A + 4) == back(g=A + 2) == -4 and back(ws=None) == back(nb=100) == back(g=A + 4, nb=0) == -5
    for dt in (B.F32, B.BF16):
        assert B.vgg_fc_xent_workspace_bytes(dt, 1, 1, 1) > 0 and B.vgg_fc_xent_bwd_workspace_bytes(dt, 1, 1, 1) > 0
        # what pieces take does not grow with the classes (but for the 8 bytes of a tile of classes that the forward pass keeps for a row)
        some, many = (B.vgg_fc_xent_bwd_workspace_bytes(dt, 8192, 2048, k) for k in (1 << 17, 1 << 20))
        assert many < 1.3 * some < 8192 * (1 << 17) * 4 / 2
    assert B.vgg_fc_xent_workspace_bytes(7, 1, 1, 1) == B.vgg_fc_xent_bwd_workspace_bytes(B.F32, 1, 0, 1) == 0
