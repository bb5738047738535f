"""Host-only checks of the entry points for answers, 4-bit weights and orthogonalised updates: arguments are refused before the
device is touched, and workspace queries cover what runs."""
from paper_1810_09868_amd import binding as B

A = 4096  # a 16-byte aligned address that is never used


def test_log_probs_are_refused_on_the_host():
    L = B.lib()
    call = lambda dt=0, N=2, K=10, ld=10, z=A, y=A, top=2, lp=A, h=A, tl=A, ti=A, st=A, ws=None, nb=0: L.vgg_log_probs(  # noqa: E731
        dt, N, K, ld, z, y, top, lp, h, tl, ti, st, ws, nb, None)
    assert call(z=None) == call(y=None) == call(lp=None) == call(tl=None) == call(top=0) == -1
    assert call(top=0, y=None, lp=None, h=None, tl=None, ti=None, st=None) == -1          # nothing is wanted
    assert call(dt=2) == -3
    assert call(N=0) == call(K=0) == call(ld=9) == call(top=11) == call(N=(1 << 23) + 1) == call(K=100, ld=100, top=65) == -2
    assert call(z=A + 2) == call(h=A + 4) == call(ti=A + 8) == -4
    assert B.vgg_log_probs_workspace_bytes(B.F32, 1, 200003, 5) > 0 and call(N=1, K=200003, ld=200003) == -5
    assert B.vgg_log_probs_workspace_bytes(B.F32, 100, 1000, 5) == 0
    assert B.vgg_log_probs_workspace_bytes(9, 1, 200003, 5) == B.vgg_log_probs_workspace_bytes(B.F32, 1, 10, 11) == 0
    back = lambda dt=1, N=2, K=10, ld=10, z=A, y=A, st=A, h=A, g=A, gh=A, dz=2 * A, ldd=10: L.vgg_log_probs_bwd(  # noqa: E731
        dt, N, K, ld, z, y, st, h, g, gh, dz, ldd, None)
    assert back(st=None) == back(dz=None) == back(g=None, gh=None) == back(y=None) == back(h=None) == -1
    assert back(dt=-1) == -3 and back(ldd=9) == back(dz=A, ldd=11) == back(N=-1) == -2 and back(dz=A + 2) == -4


def test_four_bit_layers_are_refused_on_the_host():
    L = B.lib()
    call = lambda dt=0, N=2, i=64, o=8, g=32, a=A, c=A, s=A, z=A, zd=0, ws=A, nb=1 << 40: L.vgg_fc_w4(  # noqa: E731
        dt, N, i, o, g, a, c, s, None, z, zd, 1, ws, nb, None)
    assert call(a=None) == call(c=None) == call(s=None) == call(z=None) == -1
    assert call(dt=3) == call(zd=3) == -3
    assert call(N=0) == call(i=0) == call(o=-1) == call(g=16) == call(i=(1 << 22) + 1) == -2
    assert call(c=A + 4) == -4
    assert B.vgg_fc_w4_workspace_bytes(B.BF16, 100, 4096, 4096, 64) > 0 and call(dt=1, N=100, i=4096, o=4096, nb=16) == -5
    assert B.vgg_fc_w4_workspace_bytes(B.BF16, 1, 25088, 4096, 64) == 0      # one row streams past the codes by itself
    assert L.vgg_fc_w4_quantize(64, 8, 32, None, A, A, None) == -1 and L.vgg_fc_w4_quantize(64, 8, 33, A, A, A, None) == -2
    assert L.vgg_fc_w4_dequantize(64, 8, 32, A, A + 2, A, None) == -4


def test_orthogonalised_updates_are_refused_on_the_host():
    L = B.lib()
    call = lambda dt=0, b=1, m=8, n=8, k=5, x=A, y=A, ws=A, nb=1 << 40: L.vgg_orthogonalize(dt, b, m, n, k, x, y, ws, nb, None)  # noqa: E731
    assert call(x=None) == call(y=None) == -1 and call(dt=7) == -3
    assert call(b=0) == call(m=0) == call(n=0) == call(k=0) == call(k=21) == call(m=40000, n=40000) == call(b=65536) == -2
    assert call(ws=None) == call(nb=16) == -5 and call(ws=A + 4) == call(x=A + 4) == -4
    assert L.vgg_muon_update(0, 1, 8, 8, 5, A, A, None, 0.1, 0.9, 1, 0.0, A, 1 << 40, None) == -1
    for dt in (B.F32, B.BF16):
        for shape in ((1, 1, 1), (1, 64, 576), (2, 28, 7933), (7, 512, 4608), (1, 4096, 25088), (1, 25088, 4096)):
            assert B.vgg_muon_workspace_bytes(dt, *shape) == B.vgg_orthogonalize_workspace_bytes(dt, *shape) > 0
    # transposed matrices are worked on alike
    assert B.vgg_muon_workspace_bytes(B.F32, 1, 1000, 4096) == B.vgg_muon_workspace_bytes(B.F32, 1, 4096, 1000)


def test_sizes_past_what_a_launch_holds_are_refused_on_the_host():
    L = B.lib()
    K = (1 << 30) + 1
    assert L.vgg_log_probs(0, 1, K, K, A, A, 0, A, A, None, None, A, A, 1 << 40, None) == -2
    assert L.vgg_log_probs_bwd(0, 1, K, K, A, A, A, A, A, None, 2 * A, K, None) == -2
    assert B.vgg_log_probs_workspace_bytes(B.F32, 1, K, 0) == 0 < B.vgg_log_probs_workspace_bytes(B.F32, 1, K - 1, 0)
    w4 = lambda N, i, o: L.vgg_fc_w4(0, N, i, o, 32, A, A, A, None, A, 0, 1, A, 1 << 50, None)  # noqa: E731
    assert w4((1 << 23) + 1, 1, 1) == w4(1, 1, (1 << 25) + 1) == w4(1 << 22, 1, 1 << 12) == w4(1 << 22, 1 << 12, 1) == -2
    assert L.vgg_fc_w4_quantize(1, (1 << 25) + 1, 32, A, A, A, None) == L.vgg_fc_w4_dequantize(1 << 22, 1 << 12, 32, A, A, A, None) == -2
    assert B.vgg_fc_w4_workspace_bytes(B.F32, (1 << 23) + 1, 64, 64, 32) == 0 < B.vgg_fc_w4_workspace_bytes(B.F32, 1 << 23, 64, 64, 32)


def test_a_part_of_a_longer_sequence_of_labels_is_taken():
    # (the workspace is looked at after the alignment: nothing is launched)
    L = B.lib()
    call = lambda y: L.vgg_log_probs(0, 1, 200003, 200003, A, y, 0, A, A, None, None, A, None, 0, None)  # noqa: E731
    assert call(A + 4) == call(A + 200) == -5 and call(A + 2) == -4
