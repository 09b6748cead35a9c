"""Layer norm, preference loss and orthogonalised updates refuse bad arguments before anything is enqueued.  No GPU: a call
that got as far as the CUDA runtime would return DP_ERR_CUDA here."""
import ctypes as C

import pytest
import torch

from paper_2609_40335_b200 import binding, build

if torch.cuda.is_available():                     # made-up addresses: only where nothing can run
    pytest.skip("for machines without a GPU", allow_module_level=True)

INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE, CUDA = 1, 2, 3, 4, 5
NAN, INF = float("nan"), float("inf")
A = [1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20, 6 << 20, 7 << 20, 8 << 20, 9 << 20]


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def layernorm(lib, **kw):
    a = dict(X=A[0], ldx=64, dt=1, rows=40, p=64, gain=A[1], shift=A[2], pdt=0, eps=1e-5, Y=A[3], ldy=64, H=A[4], ldh=64, mean=A[5],
             rstd=A[6], status=None)
    assert not set(kw) - set(a)
    a.update(kw)
    return lib.dp_layernorm(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(X=None), INVALID), (dict(rows=0), INVALID), (dict(rows=-4), INVALID), (dict(p=0), INVALID), (dict(ldx=63), INVALID),
    (dict(ldy=63), INVALID), (dict(ldh=63), INVALID), (dict(dt=2), INVALID), (dict(pdt=-1), INVALID), (dict(eps=-1e-5), INVALID),
    (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID), (dict(Y=A[4]), INVALID), (dict(Y=None, H=None, mean=None, rstd=None), INVALID),
    (dict(p=16385, ldx=16385, ldy=16385, ldh=16385), UNSUPPORTED), (dict(X=A[0] + 1), ALIGNMENT), (dict(mean=A[5] + 2), ALIGNMENT),
    (dict(gain=A[1] + 2), ALIGNMENT), (dict(Y=A[0], ldy=72), INVALID),
    (dict(), CUDA), (dict(X=A[0] + 2, gain=None, Y=None, mean=None), CUDA), (dict(Y=A[0]), CUDA)])
def test_layernorm(lib, kw, want):
    assert layernorm(lib, **kw) == want


def test_layernorm_of_more_rows_than_a_block_counts(lib):
    """2^36 rows on four blocks are 2^31 tiles each: counted in 32 bits, none would be read."""
    kw = dict(rows=1 << 36, p=1, ldx=1, ldy=1, ldh=1, H=None, mean=None, rstd=None)
    assert layernorm(lib, **kw) == CUDA
    before = lib.dp_set_reserved_sms(146)
    try:
        assert layernorm(lib, **kw) == UNSUPPORTED and layernorm(lib, **dict(kw, rows=1 << 35)) == CUDA
    finally:
        lib.dp_set_reserved_sms(before)


def backward(lib, **kw):
    a = dict(G=A[0], ldg=64, X=A[1], ldx=64, dt=1, B=3, T=20, p=64, gain=A[2], pdt=0, mean=A[3], rstd=A[4], dX=A[5], lddx=64, gs=A[6],
             ss=A[7], sq=A[8], ws=None, n=0, status=None)
    assert not set(kw) - set(a)
    a.update(kw)
    return lib.dp_layernorm_backward(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(G=None), INVALID), (dict(X=None), INVALID), (dict(mean=None), INVALID), (dict(rstd=None), INVALID), (dict(B=0), INVALID),
    (dict(T=0), INVALID), (dict(p=-1), INVALID), (dict(ldg=63), INVALID), (dict(ldx=63), INVALID), (dict(lddx=63), INVALID),
    (dict(dt=7), INVALID), (dict(pdt=2), INVALID), (dict(dX=None, gs=None, ss=None, sq=None), INVALID),
    (dict(p=16385, ldg=16385, ldx=16385, lddx=16385), UNSUPPORTED), (dict(B=1, T=100000), WORKSPACE),
    (dict(B=1, T=100000, ws=A[0] + 2, n=1 << 30), ALIGNMENT), (dict(G=A[0] + 1), ALIGNMENT), (dict(gs=A[6] + 2), ALIGNMENT),
    (dict(dX=A[0], lddx=72), INVALID),
    (dict(), CUDA), (dict(gain=None, dX=None, sq=None), CUDA), (dict(B=1, T=100000, gs=None, ss=None, sq=None), CUDA)])
def test_layernorm_backward(lib, kw, want):
    assert backward(lib, **kw) == want


def test_layernorm_backward_needs_a_workspace_for_few_long_examples_only(lib):
    f = lib.dp_layernorm_backward_ws_bytes
    assert f(64, 256, 768) == 0 and f(4, 16, 64) == 0 and f(6, 1024, 768) == 0
    assert f(16, 640, 776) > 0 and f(1, 4100, 1001) > 0
    assert f(1, 100000, 768) > 32 * 2 * 768 * 4 and f(0, 5, 5) == 0 and f(1, 100000, 16385) == 0


@pytest.mark.parametrize("T,want", [(1 << 30, WORKSPACE), ((1 << 30) + 1, UNSUPPORTED), ((1 << 31) - 1, UNSUPPORTED)])
def test_layernorm_backward_of_more_tokens_than_it_counts(lib, T, want):
    """Rows are counted in 32 bits, a tile or two ahead: past that no row would be read, or rows before the first."""
    kw = dict(B=1, T=T, p=1, ldg=1, ldx=1, lddx=1)
    assert backward(lib, **kw) == want
    assert (lib.dp_layernorm_backward_ws_bytes(1, T, 1) > 0) == (want == WORKSPACE)
    if want != UNSUPPORTED:
        assert backward(lib, **dict(kw, ws=A[0], n=1 << 30)) == CUDA


def preference(lib, **kw):
    a = dict(x=A[0], ldl=104, dt=1, B=3, T=20, V=100, targets=A[1], ref=A[2], beta=0.1, smoothing=0.0, scale=1.0, loss=A[3], logp=A[4],
             G=A[5], ldg=104, ws=A[6], n=1 << 20, status=A[7])
    assert not set(kw) - set(a)
    a.update(kw)
    return lib.dp_preference_loss(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), INVALID), (dict(targets=None), INVALID), (dict(B=0), INVALID), (dict(T=0), INVALID), (dict(V=0), INVALID),
    (dict(ldl=99), INVALID), (dict(ldg=99), INVALID), (dict(dt=2), INVALID), (dict(beta=-0.1), INVALID), (dict(beta=NAN), INVALID),
    (dict(smoothing=1.5), INVALID), (dict(smoothing=NAN), INVALID), (dict(scale=INF), INVALID),
    (dict(loss=None, logp=None, G=None), INVALID), (dict(G=A[0], ldg=112), INVALID), (dict(x=A[0] + 1), ALIGNMENT),
    (dict(G=A[5] + 1), ALIGNMENT), (dict(dt=0, x=A[0] + 2), ALIGNMENT), (dict(loss=A[3] + 2), ALIGNMENT), (dict(ws=None), WORKSPACE),
    (dict(n=64), WORKSPACE), (dict(ws=A[6] + 2), ALIGNMENT), (dict(B=1 << 20, T=1 << 12), UNSUPPORTED),
    (dict(), CUDA), (dict(G=A[0], ref=None, status=None), CUDA), (dict(x=A[0] + 2, G=None), CUDA)])
def test_preference_loss(lib, kw, want):
    assert preference(lib, **kw) == want


@pytest.mark.parametrize("V,want", [(1 << 30, CUDA), ((1 << 30) + 1, UNSUPPORTED), ((1 << 31) - 1, UNSUPPORTED)])
def test_preference_loss_of_more_words_than_it_counts(lib, V, want):
    """Columns are counted in 32 bits, up to a block's threads behind the row: near 2^31 that reads before it."""
    assert preference(lib, B=1, T=1, V=V, ldl=V, ldg=V) == want


def orthogonalize(lib, n=1, dt=0, out_dt=0, coefs=((3.4445, -4.7750, 2.0315),) * 5, steps=None, eps=1e-7, ws=A[2], size=1 << 30, second=None, **kw):
    arr = (binding._MatrixDesc * 2)()
    for D in arr:
        for k, v in dict(dict(M=A[0], ldm=64, out=A[1], ldo=64, p=96, d=64, scale=1.0), **kw).items():
            setattr(D, k, v)
    arr[1].M, arr[1].out = second or ((arr[0].M or 0) + (1 << 24), (arr[0].out or 0) + (1 << 24))
    flat = [c for s in coefs for c in s]
    return lib.dp_orthogonalize(arr, n, dt, out_dt, (C.c_float * max(1, len(flat)))(*flat), len(coefs) if steps is None else steps, eps, ws,
                                size, None, None)


@pytest.mark.parametrize("kw,want", [
    (dict(n=0), INVALID), (dict(dt=2), INVALID), (dict(out_dt=-1), INVALID), (dict(steps=0), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=NAN), INVALID), (dict(M=None), INVALID), (dict(out=None), INVALID), (dict(ldm=63), INVALID), (dict(ldo=63), INVALID),
    (dict(p=0), INVALID), (dict(scale=INF), INVALID), (dict(coefs=((NAN, 0, 0),)), INVALID), (dict(coefs=((2e6, 0, 0),)), INVALID),
    (dict(coefs=((30.0, 30.0, 30.0),) * 3), INVALID), (dict(M=A[0] + 2), ALIGNMENT), (dict(out=A[1] + 2), ALIGNMENT),
    (dict(dt=1, M=A[0] + 1), ALIGNMENT), (dict(ws=None), WORKSPACE), (dict(size=1000), WORKSPACE), (dict(ws=A[2] + 8), ALIGNMENT),
    (dict(p=(1 << 20) + 1), UNSUPPORTED),
    (dict(n=2, second=(A[0], A[1])), INVALID), (dict(n=2, second=(A[1], A[4])), INVALID), (dict(n=2, second=(A[3], A[0])), INVALID),
    (dict(n=2, second=(A[0], A[4])), CUDA), (dict(n=2, M=A[1]), CUDA),
    (dict(), CUDA), (dict(n=2, coefs=((1.5, -0.5, 0.0),), dt=1, out_dt=1, M=A[0] + 2, ldm=65), CUDA)])
def test_orthogonalize(lib, kw, want):
    assert orthogonalize(lib, **kw) == want


def test_orthogonalize_workspace(lib):
    arr = (binding._MatrixDesc * 2)()
    arr[0].p, arr[0].d, arr[1].p, arr[1].d = 96, 64, 64, 96
    one = lib.dp_orthogonalize_ws_bytes(arr, 1)
    assert lib.dp_orthogonalize_ws_bytes(arr, 0) == 0 and one > 8 * 96 * 64 + 8 * 64 * 64      # X twice, A and B, two fp16 terms each
    assert lib.dp_orthogonalize_ws_bytes(arr, 2) > 2 * one - 4096
    arr[1].p = 0
    assert lib.dp_orthogonalize_ws_bytes(arr, 2) == 0


def test_orthogonalize_forms(lib):
    """The sets of matrices that the GPU tests take for their form have it on a B200's 148 SMs."""
    import test_gpu_operators as T
    for name, (shapes, *forms) in T.NS_FORMS.items():
        for out, want in zip((torch.float32, torch.bfloat16), forms):
            assert T.ns_form(shapes, out) == want, (name, out)
    assert T.ns_form([(64, 256), (256, 3)], torch.float32) is None
    assert T.ns_form([(65, 256)], torch.float32) == (False, 1)
    # the linears of a GPT-2 block
    block = lambda d: [(3 * d, d), (d, d), (4 * d, d), (d, 4 * d)]
    assert T.ns_form(block(768) * 6, torch.float32) == (True, 2) and T.ns_form(block(1024) * 24, torch.bfloat16) == (True, 3)
    bad = (binding._MatrixDesc * 1)()
    f = lib.dp_debug_orthogonalize_form
    assert f(bad, 1, 0, (C.c_float * 3)(1.5, -0.5, 0.0), 1) == -1 and f(None, 1, 0, (C.c_float * 3)(), 1) == -1
    bad[0].p = bad[0].d = 8
    assert f(bad, 1, 0, (C.c_float * 3)(NAN, 0, 0), 1) == -1 and f(bad, 1, 0, (C.c_float * 3)(1.5, -0.5, 0.0), 0) == -1


def test_cpu_tensors_and_wrong_shapes_are_refused_by_the_binding():
    x = torch.zeros(2, 3, 8)
    with pytest.raises(binding.DpGhostError):
        binding.dp_layernorm(x, None, None, 1e-5, Y=torch.zeros_like(x))
    with pytest.raises(binding.DpGhostError):
        binding.dp_layernorm_backward(x, x, None, torch.zeros(6), torch.zeros(6), dX=torch.zeros_like(x))
    with pytest.raises(binding.DpGhostError):
        binding.dp_preference_loss(torch.zeros(2, 6, 8), torch.zeros(2, 2, 4, dtype=torch.int32), None, 0.1)
    with pytest.raises(binding.DpGhostError):
        binding.dp_orthogonalize([torch.zeros(4, 4)], [torch.zeros(4, 4)])
    with pytest.raises(binding.DpGhostError):
        binding.dp_orthogonalize([], [])
    for bad in (torch.zeros(6, 7), torch.zeros(5, 8), torch.zeros(6, 8).double(), torch.zeros(8, 6).t(), torch.zeros(1, 8).expand(6, 8)):
        with pytest.raises(binding.DpGhostError):
            binding._rows(bad, 6, 8, torch.float32, "t")
    assert binding._rows(torch.zeros(2, 3, 10)[:, :, :8], 6, 8, torch.float32, "t") == 10
    assert binding._rows(torch.zeros(1, 8), 1, 8, torch.float32, "t") == 8
    with pytest.raises(binding.DpGhostError):       # examples with rows between them
        binding._rows(torch.zeros(2, 4, 8)[:, :3], 6, 8, torch.float32, "t")
