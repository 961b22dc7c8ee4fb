"""Argument checks of the embedding, layer norm, orthogonalise and Muon calls: found on the host, before anything is launched (pointers are fake
and never followed)."""
import ctypes

import pytest

A, B, C_, D, E, F_, G, H = (4096 * (i + 1) for i in range(8))       # fake device addresses, 16-byte aligned
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def mxc():
    from paper_1512_01274_amd import mxc as m
    return m


def test_embedding_refusals(mxc):
    lib = mxc.raw()

    def fwd(N=5, V=7, C=9, dtype=1, tokens=A, w=B, scale=1.0, y=C_):
        return lib.mxc_embedding_fwd(N, V, C, dtype, tokens, w, scale, y, None)

    def bwd(N=5, V=7, C=9, dtype=1, tokens=A, w=B, scale=1.0, add=0, y=C_, ws=D, wn=1 << 40):
        return lib.mxc_embedding_bwd(N, V, C, dtype, tokens, w, scale, add, y, ws, wn, None)

    for call in (fwd, bwd):
        for bad in (dict(N=0), dict(V=0), dict(C=-1), dict(N=mxc.MXC_EMBEDDING_MAX_N + 1), dict(V=mxc.MXC_EMBEDDING_MAX_V + 1), dict(C=mxc.MXC_EMBEDDING_MAX_C + 1)):
            assert call(**bad) == mxc.MXC_ERR_SHAPE, bad
        for bad in (dict(dtype=2), dict(scale=NAN), dict(scale=-INF)):
            assert call(**bad) == mxc.MXC_ERR_UNSUPPORTED, bad
        for name in ("tokens", "w", "y"):
            assert call(**{name: None}) == mxc.MXC_ERR_NULL and call(**{name: A + 2}) == mxc.MXC_ERR_ALIGN
        assert call(w=A + 8) == mxc.MXC_ERR_ALIGN and call(y=A + 4) == mxc.MXC_ERR_ALIGN
    assert bwd(add=2) == mxc.MXC_ERR_UNSUPPORTED and bwd(ws=D + 8) == mxc.MXC_ERR_ALIGN
    n = ctypes.c_size_t()
    assert lib.mxc_embedding_workspace_bytes(5, 7, 9, 1, None) == mxc.MXC_ERR_NULL
    assert lib.mxc_embedding_workspace_bytes(5, 0, 9, 1, ctypes.byref(n)) == mxc.MXC_ERR_SHAPE
    assert lib.mxc_embedding_workspace_bytes(5, 7, 9, 3, ctypes.byref(n)) == mxc.MXC_ERR_UNSUPPORTED
    for N, V, C in ((1, 1, 1), (5000, 7, 9), (100000, 50257, 4096), (mxc.MXC_EMBEDDING_MAX_N, mxc.MXC_EMBEDDING_MAX_V, mxc.MXC_EMBEDDING_MAX_C)):
        need = mxc.mxc_embedding_workspace_bytes(N, V, C, 1)
        assert need % 256 == 0
        if need:
            assert bwd(N=N, V=V, C=C, wn=need - 1) == mxc.MXC_ERR_WORKSPACE and bwd(N=N, V=V, C=C, ws=None) == mxc.MXC_ERR_WORKSPACE


def test_layernorm_refusals(mxc):
    lib = mxc.raw()

    def fwd(N=5, C=9, dtype=1, x=A, gamma=B, beta=C_, eps=1e-5, y=D, stats=E):
        return lib.mxc_layernorm_fwd(N, C, dtype, x, gamma, beta, eps, y, stats, None)

    def bwd(N=5, C=9, dtype=1, x=A, gamma=B, stats=C_, dy=D, dx=E, dgamma=F_, dbeta=G, ws=H, wn=1 << 40):
        return lib.mxc_layernorm_bwd(N, C, dtype, x, gamma, stats, dy, dx, dgamma, dbeta, ws, wn, None)

    for call in (fwd, bwd):
        for bad in (dict(N=0), dict(N=-3), dict(C=0), dict(C=mxc.MXC_LAYERNORM_MAX_C + 1)):
            assert call(**bad) == mxc.MXC_ERR_SHAPE, bad
        assert call(dtype=2) == mxc.MXC_ERR_UNSUPPORTED and call(x=None) == mxc.MXC_ERR_NULL and call(x=A + 8) == mxc.MXC_ERR_ALIGN
        assert call(gamma=B + 4) == mxc.MXC_ERR_ALIGN and call(stats=B + 2) == mxc.MXC_ERR_ALIGN
    for eps in (0.0, -1e-5, 1e-39, NAN, INF):
        assert fwd(eps=eps) == mxc.MXC_ERR_UNSUPPORTED, eps
    assert fwd(y=None) == mxc.MXC_ERR_NULL and fwd(y=A + 2) == mxc.MXC_ERR_ALIGN and fwd(beta=A + 4) == mxc.MXC_ERR_ALIGN
    for name in ("stats", "dy", "dx"):
        assert bwd(**{name: None}) == mxc.MXC_ERR_NULL
    for name in ("dy", "dx", "dgamma", "dbeta", "ws"):
        assert bwd(**{name: A + 8}) == mxc.MXC_ERR_ALIGN
    n = ctypes.c_size_t()
    assert lib.mxc_layernorm_workspace_bytes(5, 7, 1, None) == mxc.MXC_ERR_NULL
    assert lib.mxc_layernorm_workspace_bytes(0, 7, 1, ctypes.byref(n)) == mxc.MXC_ERR_SHAPE
    assert lib.mxc_layernorm_workspace_bytes(5, 7, 9, ctypes.byref(n)) == mxc.MXC_ERR_UNSUPPORTED
    for N, C in ((1, 1), (128, 1000), (16384, 4096), (3, 100000), (2147483647, 8), (1, mxc.MXC_LAYERNORM_MAX_C)):
        need = mxc.mxc_layernorm_workspace_bytes(N, C, 1)
        assert need % 256 == 0
        if need:
            assert bwd(N=N, C=C, wn=need - 1) == mxc.MXC_ERR_WORKSPACE and bwd(N=N, C=C, ws=None) == mxc.MXC_ERR_WORKSPACE


def arrays(*addresses):
    return (ctypes.c_void_p * len(addresses))(*addresses)


def test_muon_refusals(mxc):
    lib = mxc.raw()
    two, most = (ctypes.c_int * 2), mxc.MXC_ORTHOGONALIZE_MAX_SIDE

    def orth(count=2, rows=two(3, 600), cols=two(4, 700), w=arrays(A, B), dtype=1, steps=5, y=arrays(C_, D), ws=H, wn=1 << 40):
        return lib.mxc_orthogonalize(count, rows, cols, w, dtype, steps, y, ws, wn, None)

    def muon(count=2, rows=two(3, 600), cols=two(4, 700), w=arrays(A, B), g=arrays(C_, D), dtype=1, m=arrays(E, F_), wb=None, lr=1e-3, mu=0.9, nesterov=1, wd=0.1, rms=0.2, gs=1.0, steps=5,
             ws=H, wn=1 << 40):
        return lib.mxc_muon_update(count, rows, cols, w, g, dtype, m, wb, lr, mu, nesterov, wd, rms, gs, steps, ws, wn, None)

    for call in (orth, muon):
        for bad in (dict(count=0), dict(count=-1), dict(count=mxc.MXC_ORTHOGONALIZE_MAX_COUNT + 1), dict(rows=two(3, 0)), dict(cols=two(-1, 3)), dict(rows=two(most + 1, 3)),
                    dict(cols=two(3, most + 1))):
            assert call(**bad) == mxc.MXC_ERR_SHAPE, bad
        for bad in (dict(dtype=2), dict(steps=0), dict(steps=mxc.MXC_ORTHOGONALIZE_MAX_STEPS + 1)):
            assert call(**bad) == mxc.MXC_ERR_UNSUPPORTED, bad
        for bad in (dict(rows=None), dict(cols=None), dict(w=None), dict(w=arrays(A, None))):
            assert call(**bad) == mxc.MXC_ERR_NULL, bad
        assert call(w=arrays(A, B + 4)) == mxc.MXC_ERR_ALIGN and call(ws=H + 8) == mxc.MXC_ERR_ALIGN
        need = mxc.mxc_orthogonalize_workspace_bytes([3, 600], [4, 700])
        assert need and need % 256 == 0 and call(wn=need - 1) == mxc.MXC_ERR_WORKSPACE and call(ws=None) == mxc.MXC_ERR_WORKSPACE
    assert orth(y=None) == mxc.MXC_ERR_NULL and orth(y=arrays(None, A)) == mxc.MXC_ERR_NULL and orth(y=arrays(A + 2, B)) == mxc.MXC_ERR_ALIGN
    for bad in (dict(mu=1.0), dict(mu=-0.1), dict(mu=NAN), dict(nesterov=2), dict(rms=-1.0), dict(rms=NAN), dict(rms=INF), dict(lr=NAN), dict(lr=INF), dict(lr=1e37), dict(wd=NAN), dict(gs=INF)):
        assert muon(**bad) == mxc.MXC_ERR_UNSUPPORTED, bad
    for bad in (dict(g=None), dict(m=None), dict(g=arrays(A, None)), dict(m=arrays(None, A)), dict(wb=arrays(A, None))):
        assert muon(**bad) == mxc.MXC_ERR_NULL, bad
    for bad in (dict(g=arrays(A + 2, B)), dict(m=arrays(A, B + 8)), dict(wb=arrays(A + 2, B))):
        assert muon(**bad) == mxc.MXC_ERR_ALIGN, bad
    # a matrix twice among those that are written: small ones too, which need no workspace
    for sides in (dict(), dict(rows=two(3, 3), cols=two(4, 4))):
        assert orth(y=arrays(C_, C_), **sides) == mxc.MXC_ERR_UNSUPPORTED
        for bad in (dict(w=arrays(A, A)), dict(m=arrays(E, E)), dict(wb=arrays(G, G))):
            assert muon(**bad, **sides) == mxc.MXC_ERR_UNSUPPORTED, bad
    # matrices that a compute unit holds need none
    assert mxc.mxc_orthogonalize_workspace_bytes([64, 1, 576], [576, 1, 64]) == 0
    assert mxc.mxc_orthogonalize_workspace_bytes([64], [577]) > 0 and mxc.mxc_orthogonalize_workspace_bytes([65], [65]) > 0
    n = ctypes.c_size_t()
    assert lib.mxc_orthogonalize_workspace_bytes(2, two(3, 5), two(4, 6), None) == mxc.MXC_ERR_NULL
    assert lib.mxc_orthogonalize_workspace_bytes(2, None, two(4, 6), ctypes.byref(n)) == mxc.MXC_ERR_NULL
    assert lib.mxc_orthogonalize_workspace_bytes(0, two(3, 5), two(4, 6), ctypes.byref(n)) == mxc.MXC_ERR_SHAPE


def test_binding_types_and_sizes(mxc):
    """Tensors of another element type than the call reads, or with fewer elements, are refused by the binding (fake device tensors: nothing is
    launched, the library finds null pointers in a call that the binding lets through)."""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    N, V, C = 4, 11, 70
    f32, bf, i32 = torch.float32, torch.bfloat16, torch.int32
    with FakeTensorMode():
        new = lambda n, dtype=f32: torch.empty(n, dtype=dtype, device="cuda")  # noqa: E731
        rows, col, stats = (N * C, bf, f32), (C, f32, bf), (2 * N, f32, torch.float64)
        calls = [
            (mxc.mxc_embedding_fwd, dict(N=N, V=V, C=C, dtype=1, scale=1.0, stream=0), dict(tokens=(N, i32, torch.int64), w=(V * C, bf, f32), y=rows)),
            (mxc.mxc_embedding_bwd, dict(N=N, V=V, C=C, dtype=1, scale=1.0, accumulate=False, stream=0), dict(tokens=(N, i32, torch.int64), dy=rows, dw=(V * C, f32, bf))),
            (mxc.mxc_layernorm_fwd, dict(N=N, C=C, dtype=1, eps=1e-5, stream=0), dict(x=rows, gamma=col, beta=col, y=rows, stats=stats)),
            (mxc.mxc_layernorm_bwd, dict(N=N, C=C, dtype=1, stream=0), dict(x=rows, gamma=col, stats=stats, dy=rows, dx=rows, dgamma=col, dbeta=col))]
        for call, plain, tensors in calls:
            good = {k: new(n, t) for k, (n, t, _) in tensors.items()}
            with pytest.raises(mxc.MxcError) as e:
                call(**plain, **good)
            assert e.value.status == mxc.MXC_ERR_NULL
            for k, (n, t, other) in tensors.items():
                with pytest.raises(ValueError, match=k):
                    call(**plain, **{**good, k: new(n - 1, t)})
                with pytest.raises(TypeError, match=k):
                    call(**plain, **{**good, k: new(n, other)})
            for bad in (dict(N=0), dict(C=-1), dict(dtype=9)):
                with pytest.raises(mxc.MxcError):
                    call(**{**plain, **bad}, **good)
        w, g, b = torch.empty(4, 5, device="cuda"), torch.empty(4, 5, device="cuda"), torch.empty(4, 5, device="cuda", dtype=bf)
        flat, h = torch.empty(20, device="cuda"), torch.empty(4, 5, device="cuda", dtype=torch.float16)
        args = (1e-3, 0.9, True, 0.1, 0.2, 1.0, 5)
        for lists, error in [((w, [g], [g], None), TypeError), (([w], [3], [g], None), TypeError), (([b], [g], [g], None), TypeError), (([w], [g], [b], None), TypeError),
                             (([w], [g], [g], [g]), TypeError), (([flat], [g], [g], None), ValueError), (([w], [g, g], [g], None), ValueError), (([w], [g[:3]], [g], None), ValueError),
                             (([w], [h], [g], None), mxc.MxcError)]:
            with pytest.raises(error):
                mxc.mxc_muon_update(*lists, *args, None, 0)
        for x, y, error in [(g, [b], TypeError), ([g], [g], TypeError), ([flat], [b], ValueError), ([g], [b, b], ValueError), ([h], [b], mxc.MxcError), ([g, b], [b, b], TypeError)]:
            with pytest.raises(error):
                mxc.mxc_orthogonalize(x, 5, y, None, 0)
    cpu = torch.empty(4, 5)
    with pytest.raises(ValueError):
        mxc.mxc_orthogonalize([cpu], 5, [cpu], None, 0)
    for call in (lambda: mxc.mxc_orthogonalize([], 5, [], None, 0), lambda: mxc.mxc_orthogonalize_workspace_bytes([], [])):
        with pytest.raises(mxc.MxcError) as e:
            call()
        assert e.value.status == mxc.MXC_ERR_SHAPE
    with pytest.raises(ValueError):
        mxc.mxc_orthogonalize_workspace_bytes([3], [3, 4])
    for bad in (3, [3.5], ["a"]):
        with pytest.raises(TypeError):
            mxc.mxc_orthogonalize_workspace_bytes(bad, bad)


def test_binding_compares_sides(mxc):
    """Every list's matrices have the sides of the first list's: as many values in other rows are refused, more dimensions than two are the first by the rest."""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    f32, bf = torch.float32, torch.bfloat16
    args = (1e-3, 0.9, True, 0.1, 0.2, 1.0, 5, None, 0)
    with FakeTensorMode():
        new = lambda *s, dtype=f32: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
        right = dict(w=[new(4, 6), new(8, 3, 5)], g=[new(4, 6), new(8, 15)], m=[new(4, 2, 3), new(8, 5, 3)], w_bf16=[new(4, 6, dtype=bf), new(8, 15, 1, dtype=bf)])
        with pytest.raises(mxc.MxcError) as e:          # (fake tensors: null pointers)
            mxc.mxc_muon_update(*right.values(), *args)
        assert e.value.status == mxc.MXC_ERR_NULL
        for name in ("g", "m", "w_bf16"):
            for i, others in ((0, [(6, 4), (2, 12), (3, 2, 4), (24, 1)]), (1, [(15, 8), (24, 5), (3, 8, 5)])):
                for other in others:
                    wrong = list(right[name])
                    wrong[i] = new(*other, dtype=right[name][i].dtype)
                    with pytest.raises(ValueError, match=name + r"\[%d\]: a matrix of" % i):
                        mxc.mxc_muon_update(*{**right, name: wrong}.values(), *args)
            with pytest.raises(mxc.MxcError) as e:      # values without rows: those of the first list's
                mxc.mxc_muon_update(*{**right, name: [new(24, dtype=right[name][0].dtype), right[name][1]]}.values(), *args)
            assert e.value.status == mxc.MXC_ERR_NULL
        for x, y in ((new(4, 6), new(6, 4, dtype=bf)), (new(3, 4, 5, dtype=bf), new(12, 5, dtype=bf)), (new(4, 6), new(1, 24, dtype=bf))):
            with pytest.raises(ValueError, match=r"y\[0\]"):
                mxc.mxc_orthogonalize([x], 5, [y], None, 0)
        with pytest.raises(mxc.MxcError) as e:
            mxc.mxc_orthogonalize([new(4, 6), new(3, 4, 5)], 5, [new(4, 2, 3, dtype=bf), new(3, 20, dtype=bf)], None, 0)
        assert e.value.status == mxc.MXC_ERR_NULL


def test_binding_sizes_past_32_bits(mxc):
    for big in (1 << 32, (1 << 32) + 5, 1 << 31, -(1 << 31) - 1):
        for call, args in ((mxc.mxc_embedding_workspace_bytes, [5, 7, 9, 1]), (mxc.mxc_layernorm_workspace_bytes, [5, 9, 1]),
                           (mxc.mxc_embedding_fwd, [5, 7, 9, 1, None, None, 1.0, None]), (mxc.mxc_layernorm_fwd, [5, 9, 1, None, None, None, 1e-5, None, None])):
            for i, a in enumerate(args):
                if isinstance(a, int):
                    with pytest.raises(OverflowError):
                        call(*args[:i], big, *args[i + 1:])
        with pytest.raises(OverflowError):
            mxc.mxc_orthogonalize_workspace_bytes([big], [5])


def test_model_refuses_other_rows():
    """Rows of another length, type or layout than the window's are refused before anything runs; what a step works with lies where the weights do."""
    import torch
    from paper_1512_01274_amd.tokens import Model, text
    model = Model(17, 12, 20, 3, device="cpu")
    assert all(t is None or t.device.type == "cpu" for t in model._of_batch(5).values())
    labels = torch.zeros(4, dtype=torch.int32)
    for rows in (torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 3, dtype=torch.int64), torch.zeros(12, dtype=torch.int32), torch.zeros(3, 4, dtype=torch.int32).t()):
        with pytest.raises(ValueError, match="rows"):
            model.train_step(rows, labels)
        with pytest.raises(ValueError, match="rows"):
            model.predict(rows)
    assert model.step == 0
    rows, labels = text(17, 3, device="cpu")(70)
    assert rows.shape == (70, 3) and labels.shape == (70,) and bool((rows[0] == -1).all()) and torch.equal(rows[1:64, -1], labels[:63])


def test_model_of_many_batch_sizes_holds_twice_the_largest(mxc):
    """What is kept for batches of all sizes is less than twice the largest's buffers and twice the largest workspace (sums of powers of two), and stays where it is; a batch of no rows is
    refused."""
    import torch
    from paper_1512_01274_amd.tokens import Model
    model = Model(17, 12, 20, 3, device="cpu")
    with pytest.raises(ValueError, match="rows"):
        model.predict(torch.zeros(0, 3, dtype=torch.int32))
    with pytest.raises(ValueError, match="rows"):
        model.train_step(torch.zeros(0, 3, dtype=torch.int32), torch.zeros(0, dtype=torch.int32))
    buffers, workspaces = {}, {}
    for N in [1, 300, *range(2, 513, 7), 300, 512, 5]:
        b = model._of_batch(N)
        for name, rows in (("e", 3 * N), ("da", 3 * N), ("s0", 3 * N), ("h", N), ("z", N), ("weight", N), ("s1", N)):
            assert b[name].shape[0] >= rows and b[name].is_contiguous()
        ws = b.pop("workspace")
        assert ws is None or ws.nbytes >= mxc.mxc_layernorm_workspace_bytes(3 * N, 12, 1)
        workspaces[0 if ws is None else ws.data_ptr()] = 0 if ws is None else ws.nbytes
        buffers.setdefault(tuple(t.data_ptr() for t in b.values()), sum(t.nbytes for t in b.values()))
        again = model._of_batch(N)
        assert again["workspace"] is ws and all(again[k] is t for k, t in b.items())
    assert sum(buffers.values()) < 2 * max(buffers.values()) and sum(workspaces.values()) < 2 * max(workspaces.values())


def test_layernorm_workspace_of_the_longest(mxc):
    """The most rows of rows that registers do not hold: two sums a row and a share of the weights' gradients, in sizes past 32 bits."""
    for C in (40000, mxc.MXC_LAYERNORM_MAX_C):
        need = [mxc.mxc_layernorm_workspace_bytes(N, C, 1) for N in (1 << 30, (1 << 31) - 4096, (1 << 31) - 1)]
        assert need == sorted(need) and need[-1] >= 8 * ((1 << 31) - 1) + 8 * C


def test_layernorm_workspace_is_of_what_a_second_launch_adds(mxc):
    """The gradient of up to 512 rows that registers hold is one launch, which leaves nothing for another."""
    for dtype in (0, 1):
        for C in (1, 100, 4097, 16384):
            assert [mxc.mxc_layernorm_workspace_bytes(N, C, dtype) for N in (1, 100, 512)] == [0, 0, 0]
            assert mxc.mxc_layernorm_workspace_bytes(513, C, dtype) > 0
        assert mxc.mxc_layernorm_workspace_bytes(1, 16385, dtype) > 0
