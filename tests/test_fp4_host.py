"""Operators in 4-bit floating point and activations, host side: refusals come before anything touches a device, so they are checked with addresses that are
never followed; and the references on cases worked by hand."""
import ctypes as C

import numpy as np
import pytest

import fp4_reference as ref
from paper_2608_00358_b200 import binding as hb
from test_experts_host import A, routing, status


def test_quantise_refusals():
    def go(x=A, ldx=64, M=4, K=64, dt=hb.BF16, fmt=hb.NVFP4, wide=1.0, r=None, q=A, ldq=32, s=A, lds=4, n=4):
        return status(hb.hccl_quantize_rows_fp4, x, ldx, M, K, dt, fmt, wide, C.byref(r) if r else None, q, ldq, s, lds, n, 0)

    assert go(fmt=2) == hb.ERR_DTYPE and go(dt=7) == hb.ERR_DTYPE
    assert go(x=0) == hb.ERR_INVALID_ARG and go(q=0) == hb.ERR_INVALID_ARG and go(s=0) == hb.ERR_INVALID_ARG
    assert go(ldx=63) == hb.ERR_INVALID_ARG and go(ldq=31) == hb.ERR_INVALID_ARG and go(lds=3) == hb.ERR_INVALID_ARG
    assert go(fmt=hb.MXFP4, lds=1) == hb.ERR_INVALID_ARG
    assert go(x=A + 1) == hb.ERR_ALIGNMENT
    assert go(n=3) == hb.ERR_COUNT_MISMATCH and go(M=-1) == hb.ERR_INVALID_ARG and go(K=-1) == hb.ERR_INVALID_ARG
    big = 1 << 20
    assert go(K=(1 << 17) + 1, ldx=big, ldq=big, lds=big) == hb.ERR_INVALID_ARG
    for wide in (0.0, -1.0, float("nan"), float("inf"), 1e-31, 1e31):
        assert go(wide=wide) == hb.ERR_INVALID_ARG, wide
    assert go(r=routing(tokens=5), n=10) == hb.ERR_COUNT_MISMATCH
    assert go(r=routing(slots=0), n=10) == hb.ERR_INVALID_ARG
    assert go(ldx=1 << 61) == hb.ERR_INVALID_ARG
    assert go(M=1 << 31, n=1 << 31) == hb.ERR_INVALID_ARG and go(n=1 << 31) == hb.ERR_INVALID_ARG


def test_dequantise_refusals():
    def go(q=A, ldq=32, s=A, lds=4, M=4, K=64, fmt=hb.NVFP4, wide=1.0, y=A, ldy=64, dt=hb.BF16):
        return status(hb.hccl_dequantize_rows_fp4, q, ldq, s, lds, M, K, fmt, wide, y, ldy, dt, 0)

    assert go(fmt=-1) == hb.ERR_DTYPE and go(dt=3) == hb.ERR_DTYPE
    assert go(q=0) == hb.ERR_INVALID_ARG and go(s=0) == hb.ERR_INVALID_ARG and go(y=0) == hb.ERR_INVALID_ARG
    assert go(ldq=31) == hb.ERR_INVALID_ARG and go(lds=3) == hb.ERR_INVALID_ARG and go(ldy=63) == hb.ERR_INVALID_ARG
    assert go(y=A + 1) == hb.ERR_ALIGNMENT and go(wide=0.0) == hb.ERR_INVALID_ARG


def test_sizes_of_laid_out_scales():
    # tiles of 128 rows, stages of 256 elements, 4 or 2 atoms of 512 bytes each
    assert hb.hccl_fp4_weight_scale_bytes(128, 256, 0, hb.NVFP4) == 2048
    assert hb.hccl_fp4_weight_scale_bytes(129, 257, 3, hb.NVFP4) == 3 * 2 * 2 * 2048
    assert hb.hccl_fp4_weight_scale_bytes(1, 1, 1, hb.MXFP4) == 1024
    assert hb.hccl_fp4_weight_scale_bytes(0, 64, 0, hb.MXFP4) == 0 and hb.hccl_fp4_weight_scale_bytes(64, 0, 0, hb.MXFP4) == 0
    for bad in ((-1, 64, 0, 0), (64, -1, 0, 0), (64, 64, -1, 0), (64, 64, 2049, 0), (64, (1 << 17) + 1, 0, 0), (1 << 31, 64, 0, 0), (1 << 28, 1 << 17, 0, 0)):
        with pytest.raises(hb.HcclError) as e:
            hb.hccl_fp4_weight_scale_bytes(*bad)
        assert e.value.status == hb.ERR_INVALID_ARG
    with pytest.raises(hb.HcclError) as e:
        hb.hccl_fp4_weight_scale_bytes(64, 64, 0, 2)
    assert e.value.status == hb.ERR_DTYPE


def test_weight_scale_refusals():
    def go(s=A, lds=4, N=8, K=64, groups=0, fmt=hb.NVFP4, out=A):
        return status(hb.hccl_fp4_weight_scales, s, lds, N, K, groups, fmt, out, 0)

    assert go(s=0) == hb.ERR_INVALID_ARG and go(out=0) == hb.ERR_INVALID_ARG and go(out=A + 8) == hb.ERR_ALIGNMENT
    assert go(lds=3) == hb.ERR_INVALID_ARG and go(fmt=9) == hb.ERR_DTYPE and go(groups=2049) == hb.ERR_INVALID_ARG
    assert go(N=0) == hb.OK and go(K=0) == hb.OK


def matmul(**kw):
    c = dict(M=4, N=8, K=64, groups=0, dtype=hb.BF16, format=hb.NVFP4, x_wide=1.0, w=A, ldw=32, w_scale=A, w_wide=A, bias=0, offsets=0, y=A, ldy=8,
             scratch=A, scratch_bytes=1 << 30, dev_status=0)
    c.update(kw)
    return hb.MatmulFp4(*c.values())


@pytest.mark.parametrize("kw,want", [
    (dict(M=-1), hb.ERR_INVALID_ARG), (dict(K=(1 << 17) + 1, ldw=1 << 18), hb.ERR_INVALID_ARG), (dict(dtype=5), hb.ERR_DTYPE), (dict(format=2), hb.ERR_DTYPE),
    (dict(groups=2), hb.ERR_INVALID_ARG), (dict(groups=1025, offsets=A), hb.ERR_INVALID_ARG), (dict(w=0), hb.ERR_INVALID_ARG), (dict(w_scale=0), hb.ERR_INVALID_ARG),
    (dict(w_wide=0), hb.ERR_INVALID_ARG), (dict(y=0), hb.ERR_INVALID_ARG), (dict(ldw=16), hb.ERR_INVALID_ARG), (dict(ldw=40), hb.ERR_ALIGNMENT),
    (dict(w=A + 8), hb.ERR_ALIGNMENT), (dict(w_scale=A + 4), hb.ERR_ALIGNMENT), (dict(scratch=A + 64), hb.ERR_ALIGNMENT), (dict(y=A + 1), hb.ERR_ALIGNMENT),
    (dict(ldy=7), hb.ERR_INVALID_ARG), (dict(w_wide=A + 2), hb.ERR_ALIGNMENT), (dict(bias=A + 2), hb.ERR_ALIGNMENT), (dict(dev_status=A + 1), hb.ERR_ALIGNMENT),
    (dict(M=1 << 31), hb.ERR_INVALID_ARG), (dict(N=1 << 31, ldy=1 << 31), hb.ERR_INVALID_ARG), (dict(x_wide=0.0), hb.ERR_INVALID_ARG),
    (dict(x_wide=float("nan")), hb.ERR_INVALID_ARG), (dict(format=hb.MXFP4, x_wide=2.0), hb.ERR_INVALID_ARG), (dict(scratch=0), hb.ERR_WORKSPACE),
    (dict(scratch_bytes=hb.hccl_fp4_scratch_bytes(4, 8, 64, 0, hb.NVFP4) - 1), hb.ERR_WORKSPACE)])
def test_product_refusals(kw, want):
    m = matmul(**kw)
    assert status(hb.hccl_linear_fp4, C.byref(m), A, 1 << 18, hb.BF16, None, 0) == want
    assert status(hb.hccl_matmul_fp4, C.byref(m), A, 1 << 17, A, 1 << 14, 0) == want


def test_linear_refusals():
    m = matmul(M=8)
    assert status(hb.hccl_linear_fp4, None, A, 64, hb.BF16, None, 0) == hb.ERR_INVALID_ARG
    assert status(hb.hccl_linear_fp4, C.byref(m), 0, 64, hb.BF16, None, 0) == hb.ERR_INVALID_ARG
    assert status(hb.hccl_linear_fp4, C.byref(m), A, 64, 4, None, 0) == hb.ERR_DTYPE
    assert status(hb.hccl_linear_fp4, C.byref(m), A, 63, hb.BF16, None, 0) == hb.ERR_INVALID_ARG
    assert status(hb.hccl_linear_fp4, C.byref(m), A, 64, hb.BF16, C.byref(routing(offsets=0)), 0) == hb.ERR_INVALID_ARG
    for q, ldq, s, lds, want in ((0, 32, A, 4, hb.ERR_INVALID_ARG), (A, 16, A, 4, hb.ERR_INVALID_ARG), (A + 8, 32, A, 4, hb.ERR_ALIGNMENT), (A, 40, A, 4, hb.ERR_ALIGNMENT),
                                 (A, 32, 0, 4, hb.ERR_INVALID_ARG), (A, 32, A, 3, hb.ERR_INVALID_ARG)):
        assert status(hb.hccl_matmul_fp4, C.byref(m), q, ldq, s, lds, 0) == want, (q, ldq, s, lds)


def experts(**kw):
    c = dict(H=64, I=32, experts=8, format=hb.NVFP4, act=hb.ACT_SILU, gated=1, up=A, ld_up=32, up_scale=A, up_wide=A, up_bias=0, down=A, ld_down=16, down_scale=A, down_wide=A, down_bias=0)
    c.update(kw)
    return hb.ExpertsFp4(*c.values())


def test_layer_refusals():
    def go(e=None, x=A, ldx=64, dt=hb.BF16, r=None, y=A, ldy=64, ws=A, n=1 << 30, st=0):
        return status(hb.hccl_expert_layer_fp4, C.byref(e or experts()), x, ldx, dt, C.byref(r or routing()), y, ldy, ws, n, st, 0)

    assert go(dt=4) == hb.ERR_DTYPE and go(e=experts(format=3)) == hb.ERR_DTYPE
    for kw in (dict(H=0), dict(I=0), dict(act=3), dict(act=-1), dict(up=0), dict(up_scale=0), dict(up_wide=0), dict(down=0), dict(down_scale=0), dict(down_wide=0),
               dict(ld_up=16), dict(ld_down=0), dict(H=(1 << 17) + 1, ld_up=1 << 17), dict(I=(1 << 17) + 1, ld_down=1 << 17)):
        assert go(e=experts(**kw), ldx=1 << 18, ldy=1 << 18) == hb.ERR_INVALID_ARG, kw
    for kw in (dict(up=A + 8), dict(ld_up=40), dict(up_scale=A + 4), dict(up_wide=A + 2), dict(up_bias=A + 1), dict(down=A + 8), dict(ld_down=24), dict(down_scale=A + 4),
               dict(down_wide=A + 2), dict(down_bias=A + 1)):
        assert go(e=experts(**kw)) == hb.ERR_ALIGNMENT, kw
    assert go(e=experts(experts=9)) == hb.ERR_COUNT_MISMATCH
    assert go(x=0) == hb.ERR_INVALID_ARG and go(y=0) == hb.ERR_INVALID_ARG and go(ldx=63) == hb.ERR_INVALID_ARG and go(ldy=63) == hb.ERR_INVALID_ARG
    assert go(x=A + 1) == hb.ERR_ALIGNMENT and go(st=A + 1) == hb.ERR_ALIGNMENT and go(ws=A + 64) == hb.ERR_ALIGNMENT
    need = hb.hccl_expert_layer_scratch_bytes(experts(), 4, 2)
    assert go(n=need - 1) == hb.ERR_WORKSPACE and go(ws=0) == hb.ERR_WORKSPACE
    assert go(r=routing(tokens=65)) == hb.ERR_INVALID_ARG and go(r=routing(tokens=-1)) == hb.ERR_INVALID_ARG
    for name in ("weights", "offsets", "slots", "source"):
        assert go(r=routing(**{name: 0})) == hb.ERR_INVALID_ARG, name
        assert go(r=routing(**{name: A + 2})) == hb.ERR_ALIGNMENT, name
    assert go(r=routing(tokens=0)) == hb.OK
    with pytest.raises(hb.HcclError):
        hb.hccl_expert_layer_scratch_bytes(experts(), 65, 2)
    with pytest.raises(hb.HcclError):
        hb.hccl_expert_layer_scratch_bytes(experts(), 4, 33)


@pytest.mark.parametrize("T,k,H,I,gated", [(1, 1, 64, 32, 1), (1, 8, 4096, 2048, 1), (64, 8, 4096, 2048, 1), (64, 32, 131072, 1000, 0), (3, 1, 131072, 131072, 1), (50, 2, 257, 129, 0), (64, 1, 1, 1, 1)])
@pytest.mark.parametrize("fmt", [hb.NVFP4, hb.MXFP4])
def test_layer_scratch_holds_every_cut_of_k(T, k, H, I, gated, fmt):
    """The first kernel cuts K by the number of units; whatever number of chunks the rows make, the partial sums fit, and beside them the pieces
    and two tiles of partial results for each block."""
    blocks, rows, halves, k_blocks = 148, T * k, 2 if gated else 1, -(-H // 256)
    width, tiles, most = halves * (-(-I // 8) * 8), halves * -(-I // 128), 0
    for filled in {1, 2, rows // 8 + 1, rows // 2 + 1, rows}:
        if filled > rows:
            continue
        for chunks in {-(-filled // 8), filled}:  # from full chunks to a row in each
            span = 4
            while span > 1 and chunks * tiles * -(-k_blocks // span) < 6 * blocks:
                span //= 2
            most = max(most, -(-k_blocks // span) * filled * width)
    need = 4 * most + rows * 8 * -(-I // 256) * 128 + 2 * blocks * T * 128 * 4 + 4 * rows * -(-I // 1024) * 2 + 4 * -(-H // 128)
    assert need <= hb.hccl_expert_layer_scratch_bytes(experts(H=H, I=I, gated=gated, format=fmt, ld_up=1 << 17, ld_down=1 << 17), T, k)


def test_activation_refusals():
    def f(**kw):
        c = dict(act=0, gated=1, p=0.1, seed=A)
        c.update(kw)
        return C.byref(hb.Activation(*c.values()))

    def go(a=None, x=A, ldx=32, M=4, I=16, dt=hb.BF16, off=0, groups=0, y=A, ldy=16):
        return status(hb.hccl_activate, a or f(), x, ldx, M, I, dt, off, groups, y, ldy, 0)

    assert go(dt=3) == hb.ERR_DTYPE
    for kw in (dict(act=3), dict(act=-1), dict(p=1.0), dict(p=-0.1), dict(p=float("nan")), dict(seed=0)):
        assert go(a=f(**kw)) == hb.ERR_INVALID_ARG, kw
    assert go(a=f(seed=A + 4)) == hb.ERR_ALIGNMENT and go(off=A + 2, groups=1) == hb.ERR_ALIGNMENT
    assert go(groups=2) == hb.ERR_INVALID_ARG and go(groups=-1) == hb.ERR_INVALID_ARG and go(M=-1) == hb.ERR_INVALID_ARG and go(I=-1) == hb.ERR_INVALID_ARG
    assert go(x=0) == hb.ERR_INVALID_ARG and go(y=0) == hb.ERR_INVALID_ARG and go(ldx=31) == hb.ERR_INVALID_ARG and go(ldy=15) == hb.ERR_INVALID_ARG
    assert go(x=A + 1) == hb.ERR_ALIGNMENT and go(y=A + 1) == hb.ERR_ALIGNMENT
    assert go(M=0, x=0, y=0) == hb.OK and go(I=0, x=0, y=0) == hb.OK
    back = lambda dy=A, lddy=16, dx=A, lddx=32: status(hb.hccl_activate_backward, f(), dy, lddy, A, 32, 4, 16, hb.BF16, 0, 0, dx, lddx, 0)  # noqa: E731
    assert back(dy=0) == hb.ERR_INVALID_ARG and back(dx=0) == hb.ERR_INVALID_ARG and back(lddy=15) == hb.ERR_INVALID_ARG and back(lddx=31) == hb.ERR_INVALID_ARG
    assert back(dy=A + 1) == hb.ERR_ALIGNMENT and back(dx=A + 1) == hb.ERR_ALIGNMENT


def test_the_references_on_cases_worked_by_hand():
    # ties go to the even code: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    x = np.array([[6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -6, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5]], dtype=np.float32)
    want = np.array([[6, 0, 1, 1, 2, 2, 4, 4, -6, 0, -1, -1, -2, -2, -4, -4]])
    for fmt in ("nvfp4", "mxfp4"):
        codes, scale = ref.quantise(x, fmt)
        assert (ref.values(codes, scale, fmt) == want).all()
    assert ref.quantise(x, "nvfp4")[1][0, 0] == 0x38 and ref.quantise(x, "mxfp4")[1][0, 0] == 127  # 1 in e4m3, and 2^0
    # the published test vectors of Philox-4x32-10 for counters and keys of all zeros and all ones
    assert ref.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert ref.philox((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert ref.E4M3[126] == 448 and ref.E4M3[1] == 2.0 ** -9 and ref.E4M3[8] == 2.0 ** -6
