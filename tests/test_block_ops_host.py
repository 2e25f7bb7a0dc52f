"""Host-side refusals of the rotary, dropout, residual-norm and 8-bit floating-point calls: every bad argument is
rejected before any launch."""
import ctypes
import math

import pytest

from paper_2607_02829_amd import abi

pytestmark = pytest.mark.cpu

FAKE = 1 << 40          # aligned, never dereferenced: validation fails first
BF, F32 = abi.SR_BF16, abi.SR_F32


def _lib():
    try:
        return abi.lib()
    except abi.SrLibraryMissing as e:
        pytest.skip(str(e))


def _rot(**kw):
    kw = dict(dict(grid=[4, 8], pairs=[6, 10]), **kw)
    fields = {k: kw.pop(k) for k in ("axes",) if k in kw}
    r = abi.SrRotary(**kw)
    for k, v in fields.items():
        setattr(r, k, v)
    return r


def _rotary(rot=None, inverse=0, dtype=BF, B=2, S=32, heads=4, hd=32, x=FAKE, ldx=128, idx=None, shared=0, y=FAKE + 64, ldy=128):
    return _lib().sr_rotary(ctypes.byref(rot) if rot is not None else ctypes.byref(_rot()), inverse, dtype, B, S, heads, hd,
                            x, ldx, idx, shared, y, ldy, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), abi.SR_EDTYPE), (dict(inverse=2), abi.SR_EINVAL), (dict(shared=2), abi.SR_EINVAL),
    (dict(B=0), abi.SR_EINVAL), (dict(S=0), abi.SR_EINVAL), (dict(heads=0), abi.SR_EINVAL), (dict(hd=0), abi.SR_EINVAL),
    (dict(S=33), abi.SR_ESHAPE),                               # more rows than tokens, without idx
    (dict(hd=30, ldx=120, ldy=120), abi.SR_ESHAPE),            # 16 pairs in 30 channels
    (dict(hd=258, ldx=2000, ldy=2000), abi.SR_EUNSUPPORTED), (dict(heads=1025, ldx=1 << 20, ldy=1 << 20), abi.SR_EUNSUPPORTED),
    (dict(ldx=127), abi.SR_ESHAPE), (dict(ldy=127), abi.SR_ESHAPE), (dict(ldx=-128), abi.SR_ESHAPE),
    (dict(x=None), abi.SR_EINVAL), (dict(y=None), abi.SR_EINVAL), (dict(x=FAKE + 1), abi.SR_EALIGN),
    (dict(dtype=F32, y=FAKE + 2), abi.SR_EALIGN), (dict(idx=FAKE + 2), abi.SR_EALIGN),
    (dict(y=FAKE, ldy=256), abi.SR_ESHAPE),                    # in place with another stride
    (dict(B=1 << 20, S=1 << 12, idx=FAKE), abi.SR_EUNSUPPORTED),
])
def test_rotary_arguments(kw, status):
    assert _rotary(**kw) == status
    assert abi.sr_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(axes=0), abi.SR_EINVAL), (dict(axes=4), abi.SR_EINVAL), (dict(layout=2), abi.SR_EINVAL),
    (dict(grid=[4, 0]), abi.SR_EINVAL), (dict(pairs=[-1, 10]), abi.SR_EINVAL), (dict(base=0.0), abi.SR_EINVAL),
    (dict(base=-3.0), abi.SR_EINVAL), (dict(base=math.inf), abi.SR_EINVAL), (dict(origin=[math.nan, 0.0]), abi.SR_EINVAL),
    (dict(step=[1.0, math.inf]), abi.SR_EINVAL), (dict(grid=[1 << 20, 1 << 12]), abi.SR_EUNSUPPORTED),
    (dict(pairs=[1, 2], freqs=[1.0, math.nan, 0.5]), abi.SR_EINVAL),
])
def test_rotary_axes(kw, status):
    assert _rotary(rot=_rot(**kw)) == status


def test_rotary_struct_wants_an_entry_per_axis():
    for bad in (dict(grid=[], pairs=[]), dict(grid=[1] * 4, pairs=[1] * 4), dict(grid=[4], pairs=[1, 2]),
                dict(grid=[4], pairs=[2], origin=[0.0, 1.0]), dict(grid=[4], pairs=[2], freqs=[1.0])):
        with pytest.raises(ValueError):
            abi.SrRotary(**bad)
    assert _lib().sr_rotary(None, 0, BF, 1, 1, 1, 32, FAKE, 32, None, 0, FAKE, 32, None) == abi.SR_EINVAL


@pytest.mark.parametrize("drop,status", [
    (dict(p=-0.1), abi.SR_EINVAL), (dict(p=1.5), abi.SR_EINVAL), (dict(p=math.nan), abi.SR_EINVAL),
    (dict(p=0.1, group=-1), abi.SR_EINVAL), (dict(p=0.1, step_dev=FAKE + 4), abi.SR_EALIGN),
])
def test_drop(drop, status):
    d = abi.SrDrop(**drop)
    assert _lib().sr_dropout(ctypes.byref(d), BF, 4, 8, FAKE, None, FAKE, None) == status
    c = _norm(drop=d)
    n = ctypes.c_size_t()
    assert _lib().sr_residual_norm_scratch_bytes(ctypes.byref(c), ctypes.byref(n)) == status


@pytest.mark.parametrize("a,status", [
    ((3, 4, 8, FAKE, None, FAKE), abi.SR_EDTYPE), ((BF, 0, 8, FAKE, None, FAKE), abi.SR_EINVAL),
    ((BF, 4, 0, FAKE, None, FAKE), abi.SR_EINVAL), ((BF, 4, 8, None, None, FAKE), abi.SR_EINVAL),
    ((BF, 4, 8, FAKE, None, None), abi.SR_EINVAL), ((BF, 4, 8, FAKE + 2, None, FAKE), abi.SR_EALIGN),
    ((BF, 4, 8, FAKE, FAKE + 8, FAKE), abi.SR_EALIGN), ((F32, 4, 8, FAKE, None, FAKE + 4), abi.SR_EALIGN),
])
def test_dropout_arguments(a, status):
    assert _lib().sr_dropout(ctypes.byref(abi.SrDrop(p=0.1)), *a, None) == status
    assert _lib().sr_dropout(None, BF, 4, 8, FAKE, None, FAKE, None) == abi.SR_EINVAL


def _norm(**kw):
    base = dict(B=2, S=3, D=64, dtype=BF, stream_dtype=F32, norm=abi.SR_NORM_LAYER, post=1, eps=1e-6, mod_stride=64)
    return abi.SrResidualNorm(**dict(base, **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=4), abi.SR_EDTYPE), (dict(dtype=F32, stream_dtype=BF), abi.SR_EDTYPE), (dict(stream_dtype=9), abi.SR_EDTYPE),
    (dict(norm=2), abi.SR_EINVAL), (dict(post=3), abi.SR_EINVAL), (dict(B=0), abi.SR_EINVAL), (dict(S=-1), abi.SR_EINVAL),
    (dict(D=0), abi.SR_EINVAL), (dict(eps=0.0), abi.SR_EINVAL), (dict(eps=math.nan), abi.SR_EINVAL),
    (dict(D=8193), abi.SR_EUNSUPPORTED), (dict(B=1 << 16, S=1 << 15), abi.SR_EUNSUPPORTED),
    (dict(B=(1 << 22) + 1, S=1), abi.SR_EUNSUPPORTED),
])
def test_residual_norm_sizes(kw, status):
    L, c, w, g = _lib(), _norm(**kw), abi.residual_norm_params(), abi.residual_norm_grads()
    n = ctypes.c_size_t()
    b = ctypes.byref
    assert L.sr_residual_norm_scratch_bytes(b(c), b(n)) == status
    assert L.sr_residual_norm_fwd(b(c), b(w), FAKE, FAKE, FAKE, FAKE, None, None, None, None) == status
    assert L.sr_residual_norm_bwd(b(c), b(w), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, b(g), FAKE, 1 << 40, None) == status


def test_residual_norm_pointers():
    L, c, w, b = _lib(), _norm(), abi.residual_norm_params(), ctypes.byref

    def fwd(x=FAKE, y=FAKE, x1=FAKE, u=FAKE, uq=None, ue=None, stats=None, w=w, c=c):
        return L.sr_residual_norm_fwd(b(c), b(w), x, y, x1, u, uq, ue, stats, None)

    for kw, status in [(dict(x=None), abi.SR_EINVAL), (dict(x1=None), abi.SR_EINVAL), (dict(uq=FAKE), abi.SR_EINVAL),
                       (dict(ue=FAKE), abi.SR_EINVAL), (dict(y=None, u=None), abi.SR_EINVAL),
                       (dict(x=FAKE + 4), abi.SR_EALIGN), (dict(y=FAKE + 2), abi.SR_EALIGN), (dict(x1=FAKE + 8), abi.SR_EALIGN),
                       (dict(u=FAKE + 8), abi.SR_EALIGN), (dict(stats=FAKE + 4), abi.SR_EALIGN),
                       (dict(uq=FAKE + 1, ue=FAKE), abi.SR_EALIGN),
                       (dict(w=abi.residual_norm_params(post_w=FAKE + 8)), abi.SR_EALIGN),
                       (dict(w=abi.residual_norm_params(scale=FAKE + 2)), abi.SR_EALIGN),
                       (dict(w=abi.residual_norm_params(gate=FAKE), c=_norm(mod_stride=63)), abi.SR_ESHAPE)]:
        assert fwd(**kw) == status, kw
    assert L.sr_residual_norm_fwd(None, b(w), FAKE, FAKE, FAKE, FAKE, None, None, None, None) == abi.SR_EINVAL
    assert L.sr_residual_norm_fwd(b(c), None, FAKE, FAKE, FAKE, FAKE, None, None, None, None) == abi.SR_EINVAL

    def bwd(x1=FAKE, y=FAKE, stats=FAKE, dx1=FAKE, du=FAKE, dx=FAKE, dy=FAKE, g=abi.residual_norm_grads(), scratch=FAKE,
            n=1 << 40, c=c):
        return L.sr_residual_norm_bwd(b(c), b(w), x1, y, stats, dx1, du, dx, dy, b(g), scratch, n, None)

    need = abi.sr_residual_norm_scratch_bytes(c)
    for kw, status in [(dict(dx1=None, du=None), abi.SR_EINVAL), (dict(dy=None), abi.SR_EINVAL), (dict(y=None), abi.SR_EINVAL),
                       (dict(x1=None), abi.SR_EINVAL), (dict(stats=None), abi.SR_EINVAL), (dict(dx=None), abi.SR_EINVAL),
                       (dict(stats=None, du=None), abi.SR_EINVAL), (dict(scratch=None), abi.SR_EINVAL),
                       (dict(n=need - 1), abi.SR_EWORKSPACE), (dict(dx=FAKE + 4), abi.SR_EALIGN),
                       (dict(g=abi.residual_norm_grads(gate=FAKE + 4)), abi.SR_EALIGN)]:
        assert bwd(**kw) == status, kw


def test_residual_norm_scratch_is_small():
    # parts of four column sums: no more than 1024 workgroups, unless there are more samples
    for B, S, D in ((1, 16200, 1024), (8, 512, 1024), (1, 1, 8192), (2000, 3, 64)):
        assert abi.sr_residual_norm_scratch_bytes(_norm(B=B, S=S, D=D)) <= max(1024, B) * 16 * D


@pytest.mark.parametrize("a,status", [
    ((2, BF, 4, 64, FAKE, 64, FAKE, FAKE, None, None), abi.SR_EINVAL), ((0, 8, 4, 64, FAKE, 64, FAKE, FAKE, None, None), abi.SR_EDTYPE),
    ((0, BF, 0, 64, FAKE, 64, FAKE, FAKE, None, None), abi.SR_EINVAL), ((1, BF, 4, 64, FAKE, 63, FAKE, FAKE, None, None), abi.SR_ESHAPE),
    ((0, BF, 4, 64, None, 64, FAKE, FAKE, None, None), abi.SR_EINVAL), ((0, BF, 4, 64, FAKE + 1, 64, FAKE, FAKE, None, None), abi.SR_EALIGN),
    ((0, BF, 4, 64, FAKE, 64, None, None, None, None), abi.SR_EINVAL), ((0, BF, 4, 64, FAKE, 64, FAKE, None, None, None), abi.SR_EINVAL),
    ((0, BF, 4, 64, FAKE, 64, FAKE, FAKE, FAKE, None), abi.SR_EINVAL), ((0, BF, 4, 64, FAKE, 64, FAKE + 8, FAKE, None, None), abi.SR_EALIGN),
    ((0, BF, 1 << 24, 128, FAKE, 128, FAKE, FAKE, None, None), abi.SR_EUNSUPPORTED),     # 2 GiB of codes
    ((0, BF, 1 << 24, 1, FAKE, 1, FAKE, FAKE, None, None), abi.SR_EUNSUPPORTED),         # rows are whole blocks
])
def test_quantize_f8_arguments(a, status):
    assert _lib().sr_quantize_f8(*a, None) == status


@pytest.mark.parametrize("M,N,K,status", [
    (0, 8, 64, abi.SR_EINVAL), (4, 0, 64, abi.SR_EINVAL), (4, 8, 0, abi.SR_EINVAL), (4, 8, (1 << 24) + 1, abi.SR_EUNSUPPORTED),
    (1 << 24, 8, 100, abi.SR_EUNSUPPORTED), (8, 1 << 24, 128, abi.SR_EUNSUPPORTED),
])
def test_linear_f8_sizes(M, N, K, status):
    n = ctypes.c_size_t()
    assert _lib().sr_linear_f8_scratch_bytes(M, N, K, ctypes.byref(n)) == status
    assert _lib().sr_linear_f8(BF, 0, M, N, K, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, 1 << 40, None) == status


def test_linear_f8_arguments():
    L = _lib()

    def call(dtype=BF, act=0, M=4, N=8, K=64, xq=FAKE, xe=FAKE, wq=FAKE, we=FAKE, bias=None, y=FAKE, scratch=FAKE, n=1 << 40):
        return L.sr_linear_f8(dtype, act, M, N, K, xq, xe, wq, we, bias, y, scratch, n, None)

    assert call(dtype=2) == abi.SR_EDTYPE and call(act=2) == abi.SR_EINVAL
    for k in ("xq", "xe", "wq", "we", "y"):
        assert call(**{k: None}) == abi.SR_EINVAL and call(**{k: FAKE + 8}) == abi.SR_EALIGN
    assert call(bias=FAKE + 4) == abi.SR_EALIGN
    assert call(dtype=F32, M=1 << 15, N=1 << 14, K=64) == abi.SR_EUNSUPPORTED   # 2 GiB of results
    need = abi.sr_linear_f8_scratch_bytes(64, 64, 1 << 20)
    if need:
        assert call(M=64, N=64, K=1 << 20, n=need - 1) == abi.SR_EWORKSPACE
        assert call(M=64, N=64, K=1 << 20, scratch=None) == abi.SR_EINVAL
