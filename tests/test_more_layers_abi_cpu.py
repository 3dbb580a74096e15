"""Host-side checks of the embedding's, the cross entropy's and the gated linear layer's
C-ABI (no GPU needed): invalid arguments are rejected before the device is touched."""
import pytest

INVALID, NOT_SUPPORTED = 1, 2
FAKE = 1 << 40  # a non-null address that is never dereferenced
GIB = 1 << 30


@pytest.fixture(scope="module")
def lib():
    from paper_2507_23387_amd import binding

    return binding


def test_embedding_validation(lib):
    I, W, Y = (FAKE + i * GIB for i in range(3))

    def call(n=4, v=9, cols=8, dtype=0, I=I, bits=64, W=W, ldw=8, scale=1.0, Y=Y, ldy=8):
        return lib.sgemm_cube_embedding(n, v, cols, dtype, I, bits, W, ldw, scale, Y, ldy, 0)

    for kw in (dict(n=-1), dict(v=-1), dict(cols=-1), dict(dtype=3), dict(dtype=-1), dict(bits=16),
               dict(bits=0), dict(ldw=7), dict(ldy=7), dict(I=None), dict(W=None), dict(Y=None),
               dict(I=I + 4), dict(I=I + 2, bits=32), dict(W=W + 2), dict(Y=Y + 2),
               dict(Y=Y + 1, dtype=1), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(Y=W), dict(Y=W + 32), dict(Y=I), dict(Y=I - 64), dict(n=1 << 60, ldy=1 << 10)):
        assert call(**kw) == INVALID, kw
    far = dict(Y=FAKE << 1, W=FAKE << 2)
    assert call(n=(1 << 27) + 1, **far) == NOT_SUPPORTED
    assert call(v=(1 << 28) + 1, **far) == NOT_SUPPORTED
    assert call(cols=(1 << 28) + 1, ldw=1 << 29, ldy=1 << 29, **far) == NOT_SUPPORTED
    assert call(n=0, I=None, Y=None) == 0 and call(cols=0, W=None, Y=None) == 0


def test_embedding_backward_validation(lib):
    DY, I, DW, WS = (FAKE + i * GIB for i in range(4))
    need = lib.sgemm_cube_embedding_backward_workspace_size(4, 8)
    assert need > 0 and need % 256 == 0
    for sizes in ((0, 8), (4, 0), (-1, 8), (4, -1), ((1 << 27) + 1, 8)):
        assert lib.sgemm_cube_embedding_backward_workspace_size(*sizes) == 0

    def call(n=4, v=9, cols=8, dtype=2, DY=DY, lddy=8, I=I, bits=32, scale=1.0, add=0, DW=DW,
             lddw=8, WS=WS, size=need):
        return lib.sgemm_cube_embedding_backward(n, v, cols, dtype, DY, lddy, I, bits, scale, add,
                                                 DW, lddw, WS, size, 0)

    for kw in (dict(n=-1), dict(v=-1), dict(cols=-1), dict(dtype=4), dict(bits=8), dict(lddy=7),
               dict(lddw=7), dict(DY=None), dict(I=None), dict(DW=None), dict(DY=DY + 1),
               dict(DW=DW + 2), dict(I=I + 2), dict(I=I + 4, bits=64), dict(scale=float("nan")),
               dict(DW=DY), dict(DW=I), dict(DW=WS), dict(WS=None), dict(WS=WS + 8),
               dict(size=need - 1), dict(WS=DY), dict(WS=I)):
        for add in (0, 1):
            assert call(**kw, add=add) == INVALID, kw
    assert call(v=(1 << 28) + 1, DW=FAKE << 1) == NOT_SUPPORTED
    assert call(v=0, DW=None) == 0 and call(cols=0, DY=None, DW=None, WS=None, size=0) == 0


def test_cross_entropy_validation(lib):
    X, W, B, T, L, E, WS = (FAKE + i * GIB for i in range(7))
    need = lib.sgemm_cube_linear_cross_entropy_workspace_size(4, 6, 8)
    assert need > 0 and need % 256 == 0
    assert lib.sgemm_cube_linear_cross_entropy_workspace_size(0, 6, 8) == 0
    assert lib.sgemm_cube_linear_cross_entropy_workspace_size(4, -6, 8) == 0

    def call(M=4, V=6, K=8, X=X, ldx=8, W=W, ldw=None, t=0, B=B, T=T, bits=64, L=L, E=E,
             scale=2048.0, order=0, WS=WS, n=need):
        ldw = max(K if t else V, 1) if ldw is None else ldw
        return lib.sgemm_cube_linear_cross_entropy(M, V, K, X, ldx, W, ldw, t, B, T, bits, L, E,
                                                   scale, order, WS, n, 0)

    for kw in (dict(M=-1), dict(V=-1), dict(K=-1), dict(ldx=7), dict(ldw=5), dict(t=1, ldw=7),
               dict(X=None), dict(W=None), dict(T=None), dict(L=None), dict(E=None),
               dict(X=X + 2), dict(B=B + 1), dict(T=T + 4), dict(bits=16), dict(L=L + 2),
               dict(E=E + 1), dict(scale=3.0), dict(order=3), dict(L=X), dict(L=W), dict(L=B),
               dict(L=T), dict(L=E + 8), dict(E=X), dict(E=T), dict(WS=None), dict(WS=WS + 8),
               dict(n=need - 1), dict(WS=X), dict(WS=L), dict(WS=T), dict(M=1 << 29, ldx=1 << 40)):
        assert call(**kw) == INVALID, kw
    assert call(K=(1 << 30) + 1, ldx=1 << 31, W=FAKE << 3) == NOT_SUPPORTED
    assert call(M=0) == 0 and call(M=0, X=None, T=None, L=None, E=None, WS=None, n=0) == 0


def test_cross_entropy_backward_validation(lib):
    G, H, X, W, B, T, E, DX, DW, DB, WS = (FAKE + i * GIB for i in range(11))
    need = lib.sgemm_cube_linear_cross_entropy_backward_workspace_size(4, 6, 8)
    assert need > 0 and need % 256 == 0
    assert lib.sgemm_cube_linear_cross_entropy_backward_workspace_size(4, 6, -1) == 0

    def call(M=4, V=6, K=8, G=G, H=H, X=X, ldx=8, W=W, ldw=None, t=0, B=B, T=T, bits=32, E=E,
             DX=DX, lddx=8, DW=DW, lddw=None, DB=DB, scale=2048.0, order=1, WS=WS, n=need):
        ldw = max(K if t else V, 1) if ldw is None else ldw
        lddw = max(K if t else V, 1) if lddw is None else lddw
        return lib.sgemm_cube_linear_cross_entropy_backward(
            M, V, K, G, H, X, ldx, W, ldw, t, B, T, bits, E, DX, lddx, DW, lddw, DB, scale, order,
            WS, n, 0)

    for kw in (dict(M=-1), dict(ldx=7), dict(ldw=5), dict(t=1, lddw=7), dict(lddx=7), dict(G=None),
               dict(E=None), dict(X=None), dict(W=None), dict(T=None), dict(G=G + 2), dict(H=H + 1),
               dict(E=E + 2), dict(DB=DB + 3), dict(bits=7), dict(scale=0.0), dict(order=-1),
               dict(DX=X), dict(DX=G), dict(DX=T), dict(DW=W), dict(DW=DX), dict(DB=DW),
               dict(DB=B), dict(DB=E), dict(DW=H), dict(WS=None), dict(n=need - 1),
               dict(WS=WS + 16), dict(WS=E), dict(DX=WS), dict(DB=WS)):
        assert call(**kw) == INVALID, kw
    assert call(M=(1 << 30) + 1, X=FAKE << 3, DX=FAKE << 4, T=FAKE << 1) == NOT_SUPPORTED


def test_gated_validation(lib):
    X, WG, WU, BG, BU, Y, G, U, WS = (FAKE + i * GIB for i in range(9))
    need = lib.sgemm_cube_gated_linear_workspace_size(4, 6, 8)
    assert need > 0 and need % 256 == 0
    assert lib.sgemm_cube_gated_linear_workspace_size(0, 6, 8) == 0
    assert lib.sgemm_cube_gated_linear_workspace_size(4, -6, 8) == 0
    assert lib.sgemm_cube_gated_linear_workspace_size(4, 1 << 62, 8) == 0

    def call(M=4, N=6, K=8, X=X, ldx=8, WG=WG, ldg=None, WU=WU, ldu=None, t=0, BG=BG, BU=BU, act=4,
             Y=Y, ldy=6, G=G, zg=6, U=U, zu=6, scale=2048.0, order=0, WS=WS, n=need):
        ldg, ldu = (max(K if t else N, 1) if ld is None else ld for ld in (ldg, ldu))
        return lib.sgemm_cube_gated_linear(M, N, K, X, ldx, WG, ldg, WU, ldu, t, BG, BU, act, Y,
                                           ldy, G, zg, U, zu, scale, order, WS, n, 0)

    for kw in (dict(M=-1), dict(N=-1), dict(K=-1), dict(ldx=7), dict(ldg=5), dict(ldu=5),
               dict(t=1, ldu=7), dict(ldy=5), dict(zg=5), dict(zu=5), dict(X=None), dict(WG=None),
               dict(WU=None), dict(Y=None), dict(G=None), dict(U=None), dict(X=X + 2),
               dict(BG=BG + 1), dict(BU=BU + 2), dict(G=G + 2), dict(act=5), dict(act=-1),
               dict(scale=3.0), dict(order=3), dict(Y=X), dict(Y=WG), dict(Y=WU), dict(Y=BG),
               dict(Y=BU), dict(Y=G), dict(G=U), dict(U=G + 24), dict(G=X), dict(U=WU),
               dict(WS=None), dict(WS=WS + 8), dict(n=need - 1), dict(WS=X), dict(WS=Y),
               dict(G=WS), dict(M=1 << 29, ldx=1 << 40)):
        assert call(**kw) == INVALID, kw
    assert call(K=(1 << 30) + 1, ldx=1 << 31, WG=FAKE << 3, WU=FAKE << 4) == NOT_SUPPORTED
    assert call(N=1 << 62, ldg=1 << 62, ldu=1 << 62, ldy=1 << 62, K=1, M=1, G=None,
                U=None) in (INVALID, NOT_SUPPORTED)
    assert call(M=0) == 0 and call(N=0) == 0 and call(M=0, X=None, Y=None, G=None, U=None) == 0


def test_gated_backward_validation(lib):
    DY, G, U, X, WG, WU, DX, DWG, DWU, DBG, DBU, WS = (FAKE + i * GIB for i in range(12))
    need = lib.sgemm_cube_gated_linear_backward_workspace_size(4, 6, 8)
    assert need > 0 and need % 256 == 0
    assert lib.sgemm_cube_gated_linear_backward_workspace_size(4, 6, -1) == 0

    def call(M=4, N=6, K=8, DY=DY, lddy=6, G=G, ldg=6, U=U, ldu=6, X=X, ldx=8, WG=WG, WU=WU, t=0,
             act=2, DX=DX, lddx=8, DWG=DWG, lddwg=None, DWU=DWU, lddwu=None, DBG=DBG, DBU=DBU,
             scale=2048.0, order=1, WS=WS, n=need):
        ld = max(K if t else N, 1)
        lddwg, lddwu = (ld if v is None else v for v in (lddwg, lddwu))
        return lib.sgemm_cube_gated_linear_backward(
            M, N, K, DY, lddy, G, ldg, U, ldu, X, ldx, WG, ld, WU, ld, t, act, DX, lddx, DWG, lddwg,
            DWU, lddwu, DBG, DBU, scale, order, WS, n, 0)

    for kw in (dict(M=-1), dict(lddy=5), dict(ldg=5), dict(ldu=5), dict(ldx=7), dict(lddwg=5),
               dict(t=1, lddwu=7), dict(lddx=7), dict(DY=None), dict(G=None), dict(U=None),
               dict(X=None), dict(WG=None), dict(WU=None), dict(DY=DY + 2), dict(DBG=DBG + 3),
               dict(act=5), dict(scale=0.0), dict(order=-1), dict(DX=DY), dict(DX=X), dict(DWG=WG),
               dict(DWG=DX), dict(DWU=DWG), dict(DWU=WU), dict(DBG=DWU), dict(DBU=U),
               dict(DBU=DBG + 8), dict(WS=None), dict(n=need - 1), dict(WS=WS + 16), dict(WS=DY),
               dict(DX=WS), dict(DBU=WS)):
        assert call(**kw) == INVALID, kw
    assert call(M=(1 << 30) + 1, DY=FAKE << 1, G=FAKE << 2, U=FAKE << 3, X=FAKE << 4,
                DX=FAKE << 5) == NOT_SUPPORTED


def test_exports():
    import paper_2507_23387_amd as sgc

    for name in ("embedding", "embedding_backward", "gated_linear", "gated_linear_backward",
                 "linear_cross_entropy", "linear_cross_entropy_backward"):
        assert name in sgc.__all__ and callable(getattr(sgc, name))
