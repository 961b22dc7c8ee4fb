"""Argument checks of the log-probability, 4-bit and AdamW calls: found on the host, before anything is launched (pointers are fake
and never followed)."""
import ctypes

import pytest

A, B, C_, D, E, F_, G, H = (4096 * (i + 1) for i in range(8))       # fake device addresses, 16-byte aligned
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def mxc():
    from paper_1512_01274_amd import mxc as m
    return m


def test_logprob_refusals(mxc):
    lib = mxc.raw()

    def fwd(N=4, K=100, ld=104, dtype=1, z=A, labels=B, scale=1.0, top=5, logp=C_, entropy=D, stats=E, tl=F_, ti=G, ws=H, wn=1 << 30):
        return lib.mxc_logprob_fwd(N, K, ld, dtype, z, labels, scale, top, logp, entropy, stats, tl, ti, ws, wn, None)

    def bwd(N=4, K=100, ld=104, dtype=1, z=A, labels=B, scale=1.0, stats=C_, entropy=D, dlogp=E, dentropy=F_, dz=G):
        return lib.mxc_logprob_bwd(N, K, ld, dtype, z, labels, scale, stats, entropy, dlogp, dentropy, dz, None)

    def both(N=4, K=100, ld=104, dtype=1, z=A, labels=B, scale=1.0, dlogp=C_, dentropy=D, logp=E, entropy=F_, dz=G, ws=H, wn=1 << 30):
        return lib.mxc_logprob_fwd_bwd(N, K, ld, dtype, z, labels, scale, dlogp, dentropy, logp, entropy, dz, ws, wn, None)

    for call in (fwd, bwd, both):
        for bad in (dict(N=0), dict(N=-1), dict(K=0), dict(ld=99), dict(ld=-5)):
            assert call(**bad) == mxc.MXC_ERR_SHAPE, bad
        for bad in (dict(dtype=2), dict(dtype=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF)):
            assert call(**bad) == mxc.MXC_ERR_UNSUPPORTED, bad
        assert call(z=None) == mxc.MXC_ERR_NULL and call(labels=None) == mxc.MXC_ERR_NULL
        assert call(z=A + 8) == mxc.MXC_ERR_ALIGN and call(labels=B + 2) == mxc.MXC_ERR_ALIGN and call(entropy=D + 1) == mxc.MXC_ERR_ALIGN
    assert fwd(top=65) == mxc.MXC_ERR_SHAPE and fwd(top=-1) == mxc.MXC_ERR_SHAPE
    assert fwd(tl=None) == mxc.MXC_ERR_NULL and fwd(ti=None) == mxc.MXC_ERR_NULL
    assert bwd(stats=None) == mxc.MXC_ERR_NULL and bwd(dz=None) == mxc.MXC_ERR_NULL and bwd(entropy=None) == mxc.MXC_ERR_NULL
    assert both(dz=None) == mxc.MXC_ERR_NULL and both(dz=G + 4) == mxc.MXC_ERR_ALIGN
    n = ctypes.c_size_t()
    assert lib.mxc_logprob_workspace_bytes(1, 1, 0, 0, None) == mxc.MXC_ERR_NULL
    assert lib.mxc_logprob_workspace_bytes(1, 0, 0, 0, ctypes.byref(n)) == mxc.MXC_ERR_SHAPE
    assert lib.mxc_logprob_workspace_bytes(1, 1, 0, 65, ctypes.byref(n)) == mxc.MXC_ERR_SHAPE
    assert lib.mxc_logprob_workspace_bytes(1, 1, 7, 0, ctypes.byref(n)) == mxc.MXC_ERR_UNSUPPORTED


@pytest.mark.parametrize("N,K", [(1, 1), (1, 1 << 20), (3, 131072), (4096, 50257), (1 << 20, 7)])
def test_logprob_workspace(mxc, N, K):
    """What the size query names is what the call asks for."""
    lib = mxc.raw()
    for dtype in (0, 1):
        for top in (0, 5, 64):
            need = mxc.mxc_logprob_workspace_bytes(N, K, dtype, top)
            assert need % 256 == 0
            if need:
                assert lib.mxc_logprob_fwd(N, K, K, dtype, A, B, 1.0, top, C_, D, E, F_, G, H, 0, None) == mxc.MXC_ERR_WORKSPACE
                assert lib.mxc_logprob_fwd(N, K, K, dtype, A, B, 1.0, top, C_, D, E, F_, G, None, need, None) == mxc.MXC_ERR_WORKSPACE


def test_mxfp4_refusals(mxc):
    lib = mxc.raw()
    for call in (lib.mxc_mxfp4_quantize, lib.mxc_mxfp4_dequantize):
        assert call(0, 5, 0, A, B, C_, None) == mxc.MXC_ERR_SHAPE and call(5, -1, 0, A, B, C_, None) == mxc.MXC_ERR_SHAPE
        assert call(1 << 30, 1 << 30, 0, A, B, C_, None) == mxc.MXC_ERR_SHAPE
        assert call(5, 5, 2, A, B, C_, None) == mxc.MXC_ERR_UNSUPPORTED
        for i in range(3):
            null, off = [A, B, C_], [A, B, C_]
            null[i], off[i] = None, off[i] + 4
            assert call(5, 5, 1, *null, None) == mxc.MXC_ERR_NULL and call(5, 5, 1, *off, None) == mxc.MXC_ERR_ALIGN

    def fc(N=5, C=70, K=9, dtype=1, x=A, wc=B, ws=C_, bias=D, relu=1, y=E, w=F_, wn=1 << 30):
        return lib.mxc_mxfp4_fc_fwd(N, C, K, dtype, x, wc, ws, bias, relu, y, w, wn, None)

    for bad in (dict(N=0), dict(C=0), dict(K=-3), dict(C=1 << 30, K=1 << 30)):
        assert fc(**bad) == mxc.MXC_ERR_SHAPE, bad
    assert fc(dtype=5) == mxc.MXC_ERR_UNSUPPORTED and fc(relu=2) == mxc.MXC_ERR_UNSUPPORTED
    for name in ("x", "wc", "ws", "y"):
        assert fc(**{name: None}) == mxc.MXC_ERR_NULL and fc(**{name: A + 2}) == mxc.MXC_ERR_ALIGN
    assert fc(bias=D + 2) == mxc.MXC_ERR_ALIGN
    need = mxc.mxc_mxfp4_fc_workspace_bytes(300, 5000, 70, 1)
    assert need and fc(N=300, C=5000, K=70, wn=need - 256) == mxc.MXC_ERR_WORKSPACE and fc(N=300, C=5000, K=70, w=None) == mxc.MXC_ERR_WORKSPACE


def arrays(*addresses):
    return (ctypes.c_void_p * len(addresses))(*addresses)


def test_adamw_refusals(mxc):
    lib = mxc.raw()
    two = (ctypes.c_size_t * 2)

    def call(count=2, sizes=two(3, 5), w=arrays(A, B), g=arrays(C_, D), gt=0, m=arrays(E, F_), v=arrays(G, H), wb=None, lr=1e-3, b1=0.9, b2=0.999,
             eps=1e-8, wd=0.1, gs=1.0, step=1, bits=32):
        if bits == 32:
            return lib.mxc_adamw_update(count, sizes, w, g, gt, m, v, wb, lr, b1, b2, eps, wd, gs, step, None)
        return lib.mxc_adamw8_update(count, sizes, w, g, gt, m, wb, lr, b1, b2, eps, wd, gs, step, 1, None)

    for bits in (32, 8):
        for bad in (dict(count=0), dict(count=-1), dict(step=0), dict(sizes=two(3, (1 << 34) + 1))):
            assert call(bits=bits, **bad) == mxc.MXC_ERR_SHAPE, bad
        for bad in (dict(gt=2), dict(b1=1.0), dict(b2=1.0), dict(b1=-0.1), dict(b2=NAN), dict(eps=-1e-8), dict(eps=NAN), dict(lr=INF), dict(lr=NAN),
                    dict(wd=NAN), dict(gs=INF)):
            assert call(bits=bits, **bad) == mxc.MXC_ERR_UNSUPPORTED, bad
        for bad in (dict(sizes=None), dict(w=None), dict(g=None), dict(m=None), dict(w=arrays(A, None)), dict(wb=arrays(A, None))):
            assert call(bits=bits, **bad) == mxc.MXC_ERR_NULL, bad
        for bad in (dict(w=arrays(A, B + 4)), dict(g=arrays(C_ + 2, D)), dict(m=arrays(E, F_ + 8)), dict(wb=arrays(A + 2, B))):
            assert call(bits=bits, **bad) == mxc.MXC_ERR_ALIGN, bad
        # tensors of no values are passed over, whatever their pointers: here there is nothing else
        nothing = arrays(None, None)
        assert call(bits=bits, sizes=two(0, 0), w=nothing, g=nothing, m=nothing, v=nothing, wb=nothing) == mxc.MXC_OK
    assert call(v=None) == mxc.MXC_ERR_NULL and call(v=arrays(G, H + 1)) == mxc.MXC_ERR_ALIGN
    assert mxc.mxc_adamw8_state_bytes(0) == 0 and mxc.mxc_adamw8_state_bytes(1) == 528 and mxc.mxc_adamw8_state_bytes(257) == 1056
    with pytest.raises(mxc.MxcError):
        mxc.mxc_adamw8_state_bytes((1 << 34) + 1)


def test_binding_lists(mxc):
    """Lists that do not fit each other are refused by the binding (fake device tensors: nothing is launched)."""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    args = (1e-3, 0.9, 0.999, 1e-8, 0.1, 1.0, 1)
    with FakeTensorMode():
        w, g, h = (torch.empty(4, device="cuda") for _ in range(3))
        b = torch.empty(4, device="cuda", dtype=torch.bfloat16)
        for lists, error in [((w, [g], [g], [g], None), TypeError), (([w], [3], [g], [g], None), TypeError), (([b], [g], [g], [g], None), TypeError),
                             (([w], [g], [b], [g], None), TypeError), (([w], [g], [g], [g], [g]), TypeError)]:
            with pytest.raises(error):
                mxc.mxc_adamw_update(*lists, *args, 0)
    cpu = torch.empty(4)
    with pytest.raises(ValueError):
        mxc.mxc_adamw_update([cpu], [cpu], [cpu], [cpu], None, *args, 0)
    with pytest.raises(ValueError):
        mxc.mxc_adamw8_update([cpu], [cpu], [cpu], None, *args, 1, 0)
    with pytest.raises(mxc.MxcError) as e:
        mxc.mxc_adamw_update([], [], [], [], None, *args, 0)
    assert e.value.status == mxc.MXC_ERR_SHAPE


def test_sizes_past_a_launch(mxc):
    """More threads than one launch holds, or indexes past 31 bits, are refused before a launch."""
    lib, n, most = mxc.raw(), ctypes.c_size_t(), (1 << 31) - 1
    K = mxc.MXC_LOGPROB_MAX_K
    assert lib.mxc_logprob_workspace_bytes(1, K + 1, 0, 0, ctypes.byref(n)) == mxc.MXC_ERR_SHAPE
    assert lib.mxc_logprob_workspace_bytes(1, K, 0, 64, ctypes.byref(n)) == mxc.MXC_OK
    assert lib.mxc_logprob_fwd(1, K + 1, K + 1, 1, A, B, 1.0, 0, C_, D, E, None, None, H, 1 << 40, None) == mxc.MXC_ERR_SHAPE
    assert lib.mxc_logprob_bwd(1, K + 1, K + 1, 1, A, B, 1.0, C_, D, E, F_, G, None) == mxc.MXC_ERR_SHAPE
    assert lib.mxc_logprob_fwd_bwd(1, K + 1, K + 1, 1, A, B, 1.0, C_, D, E, F_, G, H, 1 << 40, None) == mxc.MXC_ERR_SHAPE
    for top, k in ((0, 1), (0, 100), (5, 1), (0, 5000), (0, 20000)):
        assert lib.mxc_logprob_fwd(most, k, k, 1, A, B, 1.0, top, C_, D, E, F_, G, H, 1 << 60, None) == mxc.MXC_ERR_SHAPE, (top, k)
        assert lib.mxc_logprob_fwd_bwd(most, k, k, 1, A, B, 1.0, C_, D, E, F_, G, H, 1 << 60, None) == mxc.MXC_ERR_SHAPE, k
        assert lib.mxc_logprob_bwd(most, k, k, 1, A, B, 1.0, C_, D, E, F_, G, None) == mxc.MXC_ERR_SHAPE, k
    for call in (lib.mxc_mxfp4_quantize, lib.mxc_mxfp4_dequantize):
        assert call(most, 1, 1, A, B, C_, None) == mxc.MXC_ERR_SHAPE
    for N, k in ((1, most), (20, most), (129, most - 70000000)):
        assert lib.mxc_mxfp4_fc_fwd(N, 1, k, 1, A, B, C_, D, 0, E, F_, 1 << 60, None) == mxc.MXC_ERR_SHAPE
    assert lib.mxc_mxfp4_fc_fwd(4, mxc.MXC_MXFP4_FC_MAX_C + 1, 8, 1, A, B, C_, D, 0, E, F_, 1 << 60, None) == mxc.MXC_ERR_SHAPE
    with pytest.raises(mxc.MxcError):
        mxc.mxc_mxfp4_fc_workspace_bytes(4, mxc.MXC_MXFP4_FC_MAX_C + 1, 8, 1)
    with pytest.raises(mxc.MxcError):
        mxc.mxc_adamw8_state_bytes((1 << 33) + 1)


def test_logprob_scales(mxc):
    """Any positive scale whose product with log2(e) 32 bits hold; the kernels count in powers of two."""
    lib = mxc.raw()
    off = A + 4         # a misaligned z: the checks before that one have passed
    for scale, want in ((1e-45, mxc.MXC_ERR_ALIGN), (1e-30, mxc.MXC_ERR_ALIGN), (2.35e38, mxc.MXC_ERR_ALIGN), (2.37e38, mxc.MXC_ERR_UNSUPPORTED), (3.4e38, mxc.MXC_ERR_UNSUPPORTED)):
        assert lib.mxc_logprob_fwd(4, 100, 104, 1, off, B, scale, 5, C_, D, E, F_, G, H, 1 << 30, None) == want, scale
        assert lib.mxc_logprob_bwd(4, 100, 104, 1, off, B, scale, C_, D, E, F_, G, None) == want, scale
        assert lib.mxc_logprob_fwd_bwd(4, 100, 104, 1, off, B, scale, C_, D, E, F_, G, H, 1 << 30, None) == want, scale


def test_binding_types_and_sizes(mxc):
    """Tensors of another element type than the call reads, or with fewer elements, are refused by the binding (fake device tensors: nothing is
    launched, the library finds null pointers in a call that the binding lets through)."""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode
    N, K, ld, top, C = 4, 100, 104, 5, 70
    with FakeTensorMode():
        new = lambda n, dtype=torch.float32: torch.empty(n, dtype=dtype, device="cuda")  # noqa: E731
        bf, i32, u8 = torch.bfloat16, torch.int32, torch.uint8
        # name: (elements, type, another type that is refused); bytes may be of any type that holds them
        z, row, ints = ((N - 1) * ld + K, bf, torch.float32), (N, torch.float32, torch.float64), (N, i32, torch.int64)
        codes, scales, wc, ws = (N * 48, u8, None), (N * 16, u8, None), (K * 48, u8, None), (K * 16, u8, None)
        calls = [
            (mxc.mxc_logprob_fwd, dict(N=N, K=K, ld=ld, dtype=1, scale=1.0, top=top, stream=0),
             dict(z=z, labels=ints, logp=row, entropy=row, stats=(2 * N, torch.float32, bf), top_logp=(N * top, torch.float32, bf), top_index=(N * top, i32, torch.int64))),
            (mxc.mxc_logprob_bwd, dict(N=N, K=K, ld=ld, dtype=1, scale=1.0, stream=0),
             dict(z=z, labels=ints, stats=(2 * N, torch.float32, torch.float64), entropy=row, dlogp=row, dentropy=row, dz=z)),
            (mxc.mxc_logprob_fwd_bwd, dict(N=N, K=K, ld=ld, dtype=1, scale=1.0, stream=0),
             dict(z=z, labels=ints, dlogp=row, dentropy=row, logp=row, entropy=row, dz=z)),
            (mxc.mxc_mxfp4_quantize, dict(N=N, C=C, dtype=0, stream=0), dict(x=(N * C, torch.float32, bf), codes=codes, scales=scales)),
            (mxc.mxc_mxfp4_dequantize, dict(N=N, C=C, dtype=1, stream=0), dict(y=(N * C, bf, torch.float16), codes=codes, scales=scales)),
            (mxc.mxc_mxfp4_fc_fwd, dict(N=N, C=C, K=K, dtype=1, relu=1, stream=0),
             dict(x=(N * C, bf, torch.float32), w_codes=wc, w_scales=ws, bias=(K, torch.float32, bf), y=(N * K, bf, torch.float32))),
        ]
        for call, plain, tensors in calls:
            good = {k: new(n, t) for k, (n, t, _) in tensors.items()}
            with pytest.raises(mxc.MxcError) as e:
                call(**plain, **good)
            assert e.value.status == mxc.MXC_ERR_NULL
            for k, (n, t, other) in tensors.items():
                with pytest.raises(ValueError, match=k):
                    call(**plain, **{**good, k: new(n - 1, t)})
                if other is not None:
                    with pytest.raises(TypeError, match=k):
                        call(**plain, **{**good, k: new(n, other)})
            # bad sizes and types of the call itself are the library's to refuse
            for bad in (dict(N=0), dict(N=-1), dict(dtype=9)):
                with pytest.raises(mxc.MxcError):
                    call(**{**plain, **bad}, **good)
        # a NULL where one may be
        with pytest.raises(mxc.MxcError) as e:
            mxc.mxc_logprob_fwd(N, K, ld, 1, new(z[0], bf), None, 1.0, 0, None, new(N), None, None, None, None, 0)
        assert e.value.status == mxc.MXC_ERR_NULL


def test_head_on_its_device():
    """What a step works with lies where the head's weights do."""
    from paper_1512_01274_amd.head import Head
    held = Head(64, 96, 37, device="cpu")._of_batch(48)
    assert held["workspace"] is not None
    assert all(t.device.type == "cpu" for t in held.values())


def test_binding_sizes_past_32_bits(mxc):
    """Sizes that an int does not hold are refused, not cut."""
    for big in (1 << 32, (1 << 32) + 5, 1 << 31, -(1 << 31) - 1):
        for call, args in ((mxc.mxc_logprob_workspace_bytes, [5, 100, 1, 3]), (mxc.mxc_mxfp4_fc_workspace_bytes, [5, 100, 70, 1]),
                           (mxc.mxc_mxfp4_quantize, [5, 100, 1, None, None, None]), (mxc.mxc_logprob_fwd, [5, 100, 104, 1, None, None, 1.0, 3] + [None] * 5),
                           (mxc.mxc_mxfp4_fc_fwd, [5, 100, 70, 1, None, None, None, None, 0, None])):
            for i, a in enumerate(args):
                if isinstance(a, int):
                    with pytest.raises(OverflowError):
                        call(*args[:i], big, *args[i + 1:])


def test_head_refuses_other_rows():
    """Rows of another length or type than the head's first layer reads are refused before anything runs."""
    import torch
    from paper_1512_01274_amd.head import Head, Served
    net = Head(64, 96, 37, device="cpu")
    served = Served.__new__(Served)
    served.dims = net.dims
    labels = torch.zeros(4, dtype=torch.int32)
    for x in (torch.zeros(4, 63), torch.zeros(4, 64), torch.zeros(64).bfloat16(), torch.zeros(4, 63).bfloat16(), torch.zeros(4, 65).bfloat16(), torch.zeros(2, 4, 64).bfloat16()):
        with pytest.raises(ValueError, match="rows"):
            net.train_step(x, labels)
        with pytest.raises(ValueError, match="rows"):
            served.score(x)
    assert net.step == 0
