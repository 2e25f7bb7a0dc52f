"""Host-side refusals of the eight-bit calls: every bad argument is rejected before any launch."""
import ctypes

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


@pytest.mark.parametrize("kind,dtype,M,N,status", [
    (2, BF, 4, 64, abi.SR_EINVAL), (-1, BF, 4, 64, abi.SR_EINVAL), (0, 5, 4, 64, abi.SR_EDTYPE),
    (0, BF, 0, 64, abi.SR_EINVAL), (1, BF, 4, 0, abi.SR_EINVAL), (1, F32, -3, 64, abi.SR_EINVAL),
    (0, BF, 4, 32, abi.SR_EUNSUPPORTED), (1, BF, 4, 100, abi.SR_EUNSUPPORTED),
    (0, BF, 1 << 20, 1024, abi.SR_EUNSUPPORTED),       # exactly 2 GiB
    (1, F32, 1 << 19, 1024, abi.SR_EUNSUPPORTED),
    (0, BF, 2147483647, 2147483584, abi.SR_EUNSUPPORTED),
])
def test_quantize_sizes(kind, dtype, M, N, status):
    L = _lib()
    assert L.sr_quantize8(kind, dtype, M, N, FAKE, FAKE, FAKE, None) == status
    assert L.sr_dequantize8(kind, dtype, M, N, FAKE, FAKE, FAKE, None) == status
    assert abi.sr_last_error()


def test_quantize_pointers():
    L = _lib()
    for bad, status in ((None, abi.SR_EINVAL), (FAKE + 8, abi.SR_EALIGN)):
        for k in range(3):
            p = [FAKE] * 3
            p[k] = bad
            assert L.sr_quantize8(0, BF, 4, 64, *p, None) == status
            assert L.sr_dequantize8(1, F32, 4, 64, *p, None) == status


@pytest.mark.parametrize("dtype,act,M,N,K,status", [
    (9, 0, 4, 8, 64, abi.SR_EDTYPE), (BF, 2, 4, 8, 64, abi.SR_EINVAL), (BF, 0, 0, 8, 64, abi.SR_EINVAL),
    (BF, 0, 4, 0, 64, abi.SR_EINVAL), (BF, 0, 4, 8, 0, abi.SR_EINVAL), (BF, 0, 4, 12, 64, abi.SR_EUNSUPPORTED),
    (BF, 0, 4, 8, 96, abi.SR_EUNSUPPORTED), (BF, 0, 4, 8, 65600, abi.SR_EUNSUPPORTED),
    (BF, 0, 1 << 21, 8, 1024, abi.SR_EUNSUPPORTED), (F32, 0, 1 << 19, 1024, 64, abi.SR_EUNSUPPORTED),
    (BF, 0, 1, 1 << 21, 1024, abi.SR_EUNSUPPORTED),
])
def test_linear_sizes(dtype, act, M, N, K, status):
    assert _lib().sr_linear8(dtype, act, M, N, K, FAKE, FAKE, FAKE, FAKE, None, FAKE, None) == status


def test_linear_pointers():
    L = _lib()
    for bad, status in ((None, abi.SR_EINVAL), (FAKE + 4, abi.SR_EALIGN)):
        for k in range(6):
            if k == 4 and bad is None:
                continue   # the bias is optional
            p = [FAKE] * 6
            p[k] = bad
            assert L.sr_linear8(BF, 0, 4, 8, 64, *p, None) == status, k


@pytest.mark.parametrize("dtype,M,N,K,status", [
    (3, 4, 8, 64, abi.SR_EDTYPE), (BF, 0, 8, 64, abi.SR_EINVAL), (BF, 4, 8, -64, abi.SR_EINVAL),
    (BF, 4, 4, 64, abi.SR_EUNSUPPORTED), (BF, 4, 8, 32, abi.SR_EUNSUPPORTED),
    (BF, 1, 1 << 16, 1 << 13, abi.SR_EUNSUPPORTED),    # a 2 GiB gradient
    (BF, 1 << 20, 1024, 64, abi.SR_EUNSUPPORTED), (BF, 1 << 21, 8, 1024, abi.SR_EUNSUPPORTED),
])
def test_weight_grad_sizes(dtype, M, N, K, status):
    L = _lib()
    n = ctypes.c_size_t()
    assert L.sr_weight_grad8_scratch_bytes(dtype, M, N, K, ctypes.byref(n)) == status
    assert L.sr_weight_grad8(dtype, M, N, K, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == status


def test_weight_grad_pointers_and_scratch():
    L = _lib()
    assert L.sr_weight_grad8_scratch_bytes(BF, 4, 8, 64, None) == abi.SR_EINVAL
    for bad, status in ((None, abi.SR_EINVAL), (FAKE + 2, abi.SR_EALIGN)):
        for k in range(5):
            if k == 4 and bad is None:
                continue   # db is optional
            p = [FAKE] * 5
            p[k] = bad
            assert L.sr_weight_grad8(BF, 4, 8, 64, *p, FAKE, 1 << 40, None) == status, k
    n = abi.sr_weight_grad8_scratch_bytes(BF, 16200, 1024, 1024)
    if n:
        p = [FAKE] * 5
        assert L.sr_weight_grad8(BF, 16200, 1024, 1024, *p, None, 0, None) == abi.SR_EINVAL
        assert L.sr_weight_grad8(BF, 16200, 1024, 1024, *p, FAKE, n - 1, None) == abi.SR_EWORKSPACE


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,K", [(8, 64), (256, 1024), (1024, 1024), (4096, 1024), (1024, 4096)])
def test_weight_grad_scratch_never_falls_with_tokens(dtype, N, K):
    _lib()
    last = 0
    for M in (*range(1, 600, 7), *range(600, 16400, 61)):
        n = abi.sr_weight_grad8_scratch_bytes(dtype, M, N, K)
        assert n >= last, (M, last, n)
        last = n


def test_scan_counts_lds_writes():
    # an LDS write behind a read takes its place in the counter: lgkmcnt(1) then retires the read; a write of a
    # register that a read is still filling is a hazard
    from paper_2607_02829_amd.isa_scan import kernel_hazards
    asm = """_Zkept:
\tds_read_b128 v[0:3], v9 offset:0
\tds_write_b64 v10, v[20:21] offset:0
\ts_waitcnt lgkmcnt(1)
\tv_add_u32 v11, v0, v1
.Lfunc_end0:
_Zearly:
\tds_read_b128 v[0:3], v9 offset:0
\tds_read_b128 v[4:7], v9 offset:64
\tds_write_b64 v10, v[20:21] offset:0
\ts_waitcnt lgkmcnt(2)
\tv_add_u32 v11, v0, v4
.Lfunc_end1:
_Zstore:
\tds_read_b128 v[0:3], v9 offset:0
\tds_write_b64 v10, v[2:3] offset:0
\ts_waitcnt lgkmcnt(0)
.Lfunc_end2:
"""
    assert kernel_hazards(asm) == {"_Zkept": 0, "_Zearly": 1, "_Zstore": 1}


def _cfg(**kw):
    base = dict(B=2, L=400, D=1024, H=16, F=4096, n_blocks=8, dtype=BF, kind=abi.SR_BLOCK_PRELN, ln_eps=1e-6, idx_shared=0)
    base.update(kw)
    return abi.SrConfig(**base)


def test_save8_sizes():
    _lib()
    for kind in (abi.SR_BLOCK_PRELN, abi.SR_BLOCK_ADALN):
        plain, save = _cfg(kind=kind), _cfg(kind=kind | abi.SR_BLOCK_SAVE8)
        a, b = abi.sr_workspace_bytes(plain, 400)[0], abi.sr_workspace_bytes(save, 400)[0]
        a1, b1 = (abi.sr_workspace_bytes(_cfg(kind=c.kind, n_blocks=9), 400)[0] for c in (plain, save))
        # per token and block: 10 D channels of a byte and a 32nd (12 with adaLN), and statistics, against 24 D bytes
        # and more in bf16
        assert b < a and (b1 - b) < 0.46 * (a1 - a)
        last = (0, 0)
        for S in range(1, 400):
            n = abi.sr_workspace_bytes(save, S)
            assert n[0] >= last[0] and n[1] >= last[1]
            last = n


def test_save8_refusals():
    L = _lib()
    for kind in (abi.SR_BLOCK_SAVE8 | 2, 32, abi.SR_BLOCK_SAVE8 | 32, -1):
        assert L.sr_workspace_bytes(ctypes.byref(_cfg(kind=kind)), 10, None, None) == abi.SR_EINVAL
    c = _cfg(kind=abi.SR_BLOCK_SAVE8)
    assert L.sr_attention_colsums(ctypes.byref(c), 25, FAKE, 1 << 40, 0, FAKE, None) == abi.SR_EUNSUPPORTED
    ada = _cfg(kind=abi.SR_BLOCK_ADALN | abi.SR_BLOCK_SAVE8)
    params = (abi.SrBlockParams * 8)()
    for i in range(8):
        for n in abi.PARAM_FIELDS:
            setattr(params[i], n, FAKE)
    assert L.sr_sparse_blocks_fwd(ctypes.byref(ada), 25, params, None, FAKE, FAKE + 4096, FAKE, 1 << 40, None, 0,
                                  None) == abi.SR_EINVAL   # adaLN without cond
    need = abi.sr_workspace_bytes(c, 25)[0]
    assert L.sr_sparse_blocks_fwd(ctypes.byref(c), 25, params, None, FAKE, FAKE + 4096, FAKE, need - 1, None, 0,
                                  None) == abi.SR_EWORKSPACE


def test_trunk_save8_arguments():
    from paper_2607_02829_amd import inputs
    from paper_2607_02829_amd.trunk import Trunk
    w = inputs.small("trunk_s")
    params = inputs.params_to_storage(inputs.block_params(w, 3), w.dtype)
    for kw in (dict(save8="yes"), dict(save8=True, select="attn")):
        with pytest.raises(ValueError):
            Trunk(w, (1, 1, 1), params, **kw)


def test_blocks8_refusals():
    L = _lib()
    n = ctypes.c_size_t()
    c = _cfg()
    assert L.sr_blocks8_scratch_bytes(ctypes.byref(c), 0, ctypes.byref(n)) == abi.SR_EINVAL
    assert L.sr_blocks8_scratch_bytes(ctypes.byref(c), 10, None) == abi.SR_EINVAL
    assert L.sr_blocks8_scratch_bytes(None, 10, ctypes.byref(n)) == abi.SR_EINVAL
    assert L.sr_blocks8_scratch_bytes(ctypes.byref(_cfg(B=1)), 200000, ctypes.byref(n)) == abi.SR_EUNSUPPORTED
    assert L.sr_blocks8_scratch_bytes(ctypes.byref(_cfg(n_blocks=0)), 10, ctypes.byref(n)) == abi.SR_EINVAL
    last = 0
    for S in range(1, 300):
        v = abi.sr_blocks8_scratch_bytes(c, S)
        assert v >= last
        last = v
    need = abi.sr_blocks8_scratch_bytes(c, 25)
    ada = {"w_ada", "b_ada"}
    for kind in (abi.SR_BLOCK_PRELN, abi.SR_BLOCK_ADALN):
        c = _cfg(kind=kind, n_blocks=2)
        for name in abi.PARAM8_FIELDS:
            used = not (name in ada if kind == abi.SR_BLOCK_PRELN else name.startswith("ln"))
            for bad, status in ((None, abi.SR_EINVAL), (FAKE + 8, abi.SR_EALIGN)):
                p = (abi.SrBlockParams8 * 2)()
                for i in range(2):
                    for f in abi.PARAM8_FIELDS:
                        setattr(p[i], f, FAKE)
                setattr(p[1], name, bad)
                got = L.sr_blocks8_fwd(ctypes.byref(c), 25, p, FAKE, FAKE, FAKE, FAKE, 16, None)
                assert got == (status if used else abi.SR_EWORKSPACE), (kind, name)
    assert L.sr_blocks8_fwd(ctypes.byref(c), 25, p, None, FAKE, FAKE, FAKE, need, None) != abi.SR_OK   # adaLN without cond
    assert L.sr_blocks8_fwd(ctypes.byref(_cfg()), 25, None, None, FAKE, FAKE, FAKE, need, None) == abi.SR_EINVAL


@pytest.mark.parametrize("dtype", [BF, F32])
def test_weight_grad_scratch_grows_with_the_tokens(dtype):
    _lib()
    for D in (64, 192, 320, 512, 768, 1024, 1152, 1536, 2048):
        sizes = [abi.sr_weight_grad8_scratch_bytes(dtype, M, D, D) for M in range(1, 100000, 97)
                 if M * D * (4 if dtype == F32 else 2) < 1 << 31]
        assert sizes == sorted(sizes), D
