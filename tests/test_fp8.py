"""The linear in 8-bit floating point, its quantisers and the norm with codes on the GPU, against their plain statement."""
import pytest
import torch

import paper_2508_07329_amd as haq
from tests import fp8_reference as ref
from tests.fp8_sizes import HALVES, ROWS16, STREAM, TILED

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16
EPS = 1e-5


def same_bits(a, b):
    a, b = a.cpu().contiguous(), b.cpu().contiguous()
    return a.shape == b.shape and a.dtype == b.dtype and torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def same_codes(q, want):
    """Bytes alike, but that any NaN is like any other."""
    q, want = q.cpu().view(torch.uint8), want.cpu().contiguous().view(torch.uint8)
    both = ((q & 0x7F) == 0x7F) & ((want & 0x7F) == 0x7F)
    return bool(((q == want) | both).all())


def same_scales(s, want):
    return torch.equal(s.cpu().nan_to_num(nan=-1.0), want.nan_to_num(nan=-1.0))


def weights(seed, K, N):
    w = torch.randn(K, N, generator=torch.Generator().manual_seed(seed)) * 0.02
    wq, sw = ref.weight_codes(w)
    return wq, sw, ref.pack_weight(wq).to(DEV), sw.to(DEV)


# ---- quantisers -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,K", [(1, 16), (1, 128), (3, 4096), (7, 144), (8, 2064), (9, 1040), (17, 112), (33, 14336), (257, 1024), (2, 65536)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_activation_codes(T, K, dtype):
    x = ref.rows(T + K, T, K, dtype)
    x[T // 2, : min(K, 128)] = 0.0  # a block without a magnitude
    x[:, -16:] *= 2.0 ** -9
    q, s = haq.haq_quant_act_fp8_packed(x.to(DEV))
    want_q, want_s = ref.act_codes(x.float())
    assert same_codes(ref.unpack_act(q.cpu(), T, K), want_q)
    assert torch.equal(ref.unpack_scale(s.cpu(), T, K), want_s)


def test_activation_codes_of_extreme_blocks():
    """Subnormals, the largest finite values, magnitudes on either side of the smallest that counts, infinities and NaN."""
    v = torch.zeros(9, 256)
    g = torch.randn(9, 256, generator=torch.Generator().manual_seed(3))
    v[0, :128] = g[0, :128] * 2.0 ** -24
    v[1] = g[1].sign() * 3.0e38
    v[2, :128], v[2, 128:] = 2.0 ** -100, 2.0 ** -101
    v[3] = g[3] * 2.0 ** -126
    v[4], v[4, 5] = g[4], float("inf")
    v[5], v[5, 200] = g[5], float("nan")
    v[6, 7] = float("nan")
    v[7, 3], v[7, 9] = -float("inf"), float("nan")
    v[8] = -0.0
    x = v.to(BF16)
    q, s = haq.haq_quant_act_fp8_packed(x.to(DEV))
    want_q, want_s = ref.act_codes(x.float())
    assert same_codes(ref.unpack_act(q.cpu(), 9, 256), want_q)
    assert same_scales(ref.unpack_scale(s.cpu(), 9, 256), want_s)


def test_activation_codes_leave_other_rows_and_strided_inputs_alone():
    T, K = 21, 208
    wide = ref.rows(5, T, K + 40, F16).to(DEV)
    x = wide[:, 8:8 + K]
    R = ref.padded_rows(T)
    q = torch.full((256 * R,), 0x55, dtype=torch.uint8, device=DEV)
    s = torch.full((2 * R,), -7.0, device=DEV)
    haq.haq_quant_act_fp8_packed(x, q_packed=q.view(torch.float8_e4m3fn), block_scale=s)
    want_q, want_s = ref.act_codes(x.cpu().float())
    assert same_codes(ref.unpack_act(q.cpu(), T, K), want_q) and torch.equal(ref.unpack_scale(s.cpu(), T, K), want_s)
    assert bool((q.view(-1, R, 16)[:, T:] == 0x55).all()) and bool((q.view(-1, R, 16)[K // 16:] == 0x55).all())
    assert bool((s.view(2, R)[:, T:] == -7.0).all())


@pytest.mark.parametrize("K,N", [(16, 16), (128, 128), (144, 112), (2064, 1040), (400, 4112), (4096, 256)])
def test_weight_codes(K, N):
    w = torch.randn(K, N, generator=torch.Generator().manual_seed(K + N)) * 0.02
    w[: min(K, 128), : min(N, 128)] *= 0.0 if K > 128 else 1.0
    w[-1, -1] = 1e30
    wq, sw = haq.haq_quant_weight_fp8(w.to(DEV))
    want_q, want_s = ref.weight_codes(w)
    assert same_bits(wq, want_q) and torch.equal(sw.cpu(), want_s)
    assert torch.equal(haq.haq_pack_weight(wq).cpu().view(torch.uint8), ref.pack_weight(want_q))


# ---- linear ---------------------------------------------------------------------------------------------------------
LINEAR = [(1, 16, 16), (1, 128, 128), (1, 4096, 256), (2, 144, 48), (5, 2064, 1040), (15, 272, 528), (16, 1024, 144), (17, 1040, 272), (31, 4112, 80),
          (33, 2048, 4096), (48, 528, 272), (64, 3584, 64), (65, 400, 1296), (97, 1296, 304), (128, 272, 144), (129, 784, 400), (200, 2064, 528),
          (257, 272, 272), (333, 528, 1040), (513, 1168, 784), (1030, 144, 2064)]


@pytest.mark.parametrize("T,K,N", LINEAR)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_linear(T, K, N, dtype):
    x = ref.rows(T * K + N, T, K, dtype)
    wq, sw, wp, swd = weights(T + K + N, K, N)
    xq, sx = ref.act_codes(x.float())
    relu = (T + K // 16 + N // 16) % 2 == 0
    want, bound = ref.linear(xq, sx, wq, sw, relu)
    act = haq.HAQ_ACT_RELU if relu else haq.HAQ_ACT_NONE
    y = haq.haq_fp8_linear(x.to(DEV), wp, swd, N, act)
    ref.assert_linear(y.cpu(), want, bound)
    q, s = haq.haq_quant_act_fp8_packed(x.to(DEV))
    wide = torch.full((T, N + 24), 7.0, dtype=dtype, device=DEV)  # rows with a gap between them
    haq.haq_gemm_fp8_packed(q, s, wp, swd, T, K, N, act, out=wide[:, :N])
    ref.assert_linear(wide[:, :N].cpu(), want, bound)
    assert bool((wide[:, N:] == 7.0).all())
    assert same_bits(y, haq.haq_fp8_linear(x.to(DEV), wp, swd, N, act))  # a call repeated is the same


@pytest.mark.parametrize("T,K,N", [size for shapes in (STREAM, TILED) for sizes in shapes.values() for size in sizes] + HALVES)
def test_linear_on_each_kernel(T, K, N):
    x = ref.rows(T * K + N, T, K, F16)
    wq, sw, wp, swd = weights(T + K + N, K, N)
    q, s = haq.haq_quant_act_fp8_packed(x.to(DEV))
    want, bound = ref.linear(*ref.act_codes(x.float()), wq, sw)
    wide = torch.full((T + 1, N + 8), 7.0, dtype=BF16, device=DEV)
    haq.haq_gemm_fp8_packed(q, s, wp, swd, T, K, N, out=wide[:T, :N])
    ref.assert_linear(wide[:T, :N].cpu(), want, bound)
    assert bool((wide[:T, N:] == 7.0).all()) and bool((wide[T] == 7.0).all())
    again = torch.empty((T, N), dtype=BF16, device=DEV)
    haq.haq_gemm_fp8_packed(q, s, wp, swd, T, K, N, out=again)
    assert same_bits(again, wide[:T, :N])


@pytest.mark.parametrize("T,K,N", [size for sizes in ROWS16.values() for size in sizes])
def test_linear_of_few_rows_on_each_kernel(T, K, N):
    x = ref.rows(T * K + N, T, K, BF16)
    wq, sw, wp, swd = weights(T + K + N, K, N)
    want, bound = ref.linear(*ref.act_codes(x.float()), wq, sw)
    wide = torch.full((T + 1, N + 8), 7.0, dtype=BF16, device=DEV)
    haq.haq_fp8_linear(x.to(DEV), wp, swd, N, out=wide[:T, :N])
    ref.assert_linear(wide[:T, :N].cpu(), want, bound)
    assert (wide[T] == 7).all() and (wide[:, N:] == 7).all()


@pytest.mark.parametrize("T,K,N", [(1, 400, 272), (20, 1040, 272), (100, 400, 144), (300, 656, 528)])
def test_linear_on_what_buffers_hold_behind_the_operands(T, K, N):
    """NaN codes and scales behind the last token, the last channel chunk and the last block count for nothing."""
    x = ref.rows(T, T, K, F16)
    wq, sw, wp, swd = weights(K, K, N)
    R, kb = ref.padded_rows(T), -(-K // 128)
    q = torch.full((-(-K // 64) * 64 * R,), 0x7F, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    s = torch.full((kb * R,), float("nan"), device=DEV)
    haq.haq_quant_act_fp8_packed(x.to(DEV), q_packed=q, block_scale=s)
    y = haq.haq_gemm_fp8_packed(q, s, wp, swd, T, K, N)
    ref.assert_linear(y.cpu(), *ref.linear(*ref.act_codes(x.float()), wq, sw))
    workspace = torch.full((haq.haq_fp8_linear_workspace_bytes(T, K, N),), 0x7F, dtype=torch.uint8, device=DEV)
    y = haq.haq_fp8_linear(x.to(DEV), wp, swd, N, workspace=workspace)
    ref.assert_linear(y.cpu(), *ref.linear(*ref.act_codes(x.float()), wq, sw))


@pytest.mark.parametrize("T", [3, 40, 200])
def test_linear_keeps_infinities_and_nan_to_their_rows_and_blocks(T):
    K, N = 400, 400
    x = ref.rows(T, T, K, F16)
    x[0, 17], x[2, 399] = float("inf"), float("nan")
    w = torch.randn(K, N, generator=torch.Generator().manual_seed(1)) * 0.02
    wq, sw = ref.weight_codes(w)
    for relu in (haq.HAQ_ACT_NONE, haq.HAQ_ACT_RELU):
        y = haq.haq_fp8_linear(x.to(DEV), ref.pack_weight(wq).to(DEV), sw.to(DEV), N, relu).cpu()
        bad = y.isnan().all(dim=1)
        assert bad[0] and bad[2] and not y[1].isnan().any() and not y[3:].isnan().any()
    w[5, 200] = float("nan")
    wq, sw = haq.haq_quant_weight_fp8(w.to(DEV))
    y = haq.haq_fp8_linear(x.to(DEV), haq.haq_pack_weight(wq), sw, N).cpu()
    assert y[1].isnan().nonzero().flatten().tolist() == [200]


def test_linear_overflows_to_infinity_in_binary16_only():
    T, K, N = 4, 256, 32
    x, w = torch.full((T, K), 300.0), torch.ones(K, N)
    wq, sw, = ref.weight_codes(w)
    for dtype in (F16, BF16):
        y = haq.haq_fp8_linear(x.to(dtype).to(DEV), ref.pack_weight(wq).to(DEV), sw.to(DEV), N).cpu()
        want, bound = ref.linear(*ref.act_codes(x.to(dtype).float()), wq, sw)
        ref.assert_linear(y, want, bound)
        assert bool(y.isinf().all()) == (dtype == F16)


@pytest.mark.parametrize("T", [3, 40])
def test_linear_into_the_buffer_of_its_rows(T):
    """y over x, and beside it in one matrix."""
    K, N = 528, 400
    x = ref.rows(T, T, K, F16)
    wq, sw, wp, swd = weights(9, K, N)
    want, bound = ref.linear(*ref.act_codes(x.float()), wq, sw)
    both = torch.zeros((T, K + N), dtype=F16, device=DEV)
    both[:, :K] = x.to(DEV)
    haq.haq_fp8_linear(both[:, :K], wp, swd, N, out=both[:, K:])
    ref.assert_linear(both[:, K:].cpu(), want, bound)
    assert same_bits(both[:, :K], x)
    over = x.to(DEV)
    haq.haq_fp8_linear(over, wp, swd, N, out=over[:, :N])
    ref.assert_linear(over[:, :N].cpu(), want, bound)
    assert same_bits(over[:, N:], x[:, N:])


def test_offsets_past_32_bits():
    """Codes, weights and rows of 4 GB and more: the first and the last rows and channels."""
    K, many = 1040, 4_200_016
    x = ref.rows(1, 64, K, F16)
    last = torch.cat([torch.arange(32), many - 32 + torch.arange(32)])
    big = torch.zeros((many, K), dtype=F16, device=DEV)
    big[last.to(DEV)] = x.to(DEV)
    wq, sw, wp, swd = weights(3, K, 32)
    y = haq.haq_fp8_linear(big, wp, swd, 32)
    ref.assert_linear(y[last.to(DEV)].cpu(), *ref.linear(*ref.act_codes(x.float()), wq, sw))
    assert not y[32:-32].any()
    del y
    n, _, q, s = haq.haq_rmsnorm_quant(big, torch.ones(K, device=DEV), EPS, haq.HAQ_CODES_E4M3, y=torch.empty_like(big))
    _, v = ref.norm(x, torch.ones(K), EPS)
    assert same_bits(n[last.to(DEV)], v.to(F16))
    R = ref.padded_rows(many)
    got = q.view(torch.uint8).view(-1, R, 16)[: K // 16][:, last.to(DEV)].permute(1, 0, 2).reshape(64, K)
    assert same_codes(got, ref.act_codes(v)[0])
    del n, q, s, big
    w = torch.zeros((K, many), device=DEV)
    small = torch.randn(K, 512, generator=torch.Generator().manual_seed(5)) * 0.02
    at = many // 128 * 128 - 128  # the last whole block and what is behind it
    w[:, :128], w[:, at:] = small[:, :128].to(DEV), small[:, 128:128 + many - at].to(DEV)
    wq, sw = haq.haq_quant_weight_fp8(w)
    del w
    wp = haq.haq_pack_weight(wq)
    keep = torch.cat([wq[:, :128].cpu().view(torch.uint8), wq[:, at:].cpu().view(torch.uint8)], dim=1)
    want_q, _ = ref.weight_codes(small[:, : 128 + many - at])
    assert same_codes(keep, want_q)
    scales = torch.cat([sw[:, :1], sw[:, at // 128:]], dim=1).cpu()
    del wq
    for T in (5, 40):
        x = ref.rows(T, T, K, F16)
        y = haq.haq_fp8_linear(x.to(DEV), wp, sw, many)
        want, bound = ref.linear(*ref.act_codes(x.float()), want_q, scales)
        ref.assert_linear(torch.cat([y[:, :128], y[:, at:]], dim=1).cpu(), want, bound)


def test_no_tokens():
    _, _, wp, sw = weights(1, 128, 32)
    x = torch.empty(0, 128, dtype=F16, device=DEV)
    assert haq.haq_fp8_linear(x, wp, sw, 32).shape == (0, 32)
    assert haq.haq_rmsnorm_quant(x, torch.ones(128, device=DEV), EPS)[0].shape == (0, 128)
    haq.haq_quant_act_fp8_packed(x)


# ---- norm -----------------------------------------------------------------------------------------------------------
def check_norm(x, weight, residual, codes, want_y, eps=EPS, **buffers):
    T, K = x.shape
    d = lambda t: None if t is None else t.to(DEV)
    y = torch.empty_like(x, device=DEV) if want_y else None
    y, total, q, s = haq.haq_rmsnorm_quant(d(x), d(weight), eps, codes, residual=d(residual), y=y, **buffers)
    h, v = ref.norm(x, weight, eps, residual)
    assert (total is None) == (residual is None) and (total is None or same_bits(total, h))
    assert (y is None) == (codes != haq.HAQ_CODES_NONE and not want_y) and (y is None or same_bits(y, v.to(x.dtype)))
    if codes == haq.HAQ_CODES_I8:
        want_q, want_s = ref.i8_codes(v)
        assert torch.equal(ref.unpack_act(q.cpu(), T, K).view(torch.int8), want_q) and same_scales(s[:T], want_s)
    if codes == haq.HAQ_CODES_E4M3:
        want_q, want_s = ref.act_codes(v)
        assert same_codes(ref.unpack_act(q.cpu(), T, K), want_q)
        assert torch.equal(ref.unpack_scale(s.cpu(), T, K), want_s)
    return v


@pytest.mark.parametrize("T,K", [(1, 16), (1, 4096), (2, 144), (3, 16384), (1, 65536), (2, 20496), (7, 1040), (33, 2064), (300, 272), (513, 272), (2046, 1040),
                                 (1000, 8208), (2049, 1024), (2050, 208), (2048, 4112), (2051, 8208)])
@pytest.mark.parametrize("codes", [haq.HAQ_CODES_NONE, haq.HAQ_CODES_I8, haq.HAQ_CODES_E4M3])
def test_norm(T, K, codes):
    for dtype in (F16, BF16):
        x, r = ref.rows(T + K, T, K, dtype), ref.rows(T + K + 1, T, K, dtype)
        weight = 1.0 + 0.2 * torch.randn(K, generator=torch.Generator().manual_seed(K))
        check_norm(x, weight, r, codes, dtype == BF16)
    check_norm(x, weight, None, codes, codes == haq.HAQ_CODES_NONE)


@pytest.mark.parametrize("T", [4, 700, 2100])
@pytest.mark.parametrize("codes", [haq.HAQ_CODES_NONE, haq.HAQ_CODES_I8, haq.HAQ_CODES_E4M3])
def test_norm_of_extreme_rows(T, codes):
    """Rows of zeros, of subnormals, of values whose squares overflow binary32, weights of zero and huge ones; with a residual sums of
    subnormals and sums that cancel."""
    K = 528
    weight = torch.randn(K, generator=torch.Generator().manual_seed(3))
    weight[:128], weight[200] = 0.0, 1e20
    for dtype, small, large in ((BF16, 2.0 ** -130, 2.0 ** 100), (F16, 2.0 ** -20, 2.0 ** 9)):
        x = ref.rows(1, T, K, dtype)
        x[0] = 0.0
        x[1] = (ref.rows(2, 1, K, F16)[0].float() * small).to(dtype)
        x[2] = (ref.rows(2, 1, K, F16)[0].float() * large).to(dtype)
        r = ref.rows(6, T, K, dtype)
        r[1] = (ref.rows(7, 1, K, F16)[0].float() * small).to(dtype)
        r[3] = -x[3]
        check_norm(x, weight, None, codes, True)
        check_norm(x, weight, None, codes, True, eps=1e-30)
        check_norm(x, weight, r, codes, True)


@pytest.mark.parametrize("T", [5, 700, 2100])
def test_norm_rows_with_infinities_and_nan_stay_apart(T):
    K = 272
    x = ref.rows(4, T, K, F16)
    r = ref.rows(5, T, K, F16)
    x[1, 3], x[3, 270] = float("inf"), float("nan")
    x[4, 5], r[4, 5] = 60000.0, 60000.0  # the sum overflows
    weight = torch.ones(K)
    other = [i for i in range(T) if i not in (1, 3, 4)]
    for codes in (haq.HAQ_CODES_I8, haq.HAQ_CODES_E4M3):
        y, total, q, s = haq.haq_rmsnorm_quant(x.to(DEV), weight.to(DEV), EPS, codes, residual=r.to(DEV), y=torch.empty_like(x, device=DEV))
        h, v = ref.norm(x, weight, EPS, r)
        assert same_bits(y[other], v[other].to(F16)) and y.cpu()[[1, 3, 4]].isnan().any(dim=1).all()
        if codes == haq.HAQ_CODES_I8:
            assert bool(s.cpu()[[1, 3, 4]].isfinite().logical_not().all()) and bool(s.cpu()[other].isfinite().all())
            codes_ = ref.unpack_act(q.cpu(), T, K)
            assert bool((codes_[[1, 3, 4]] == 0).all()) and torch.equal(codes_[other].view(torch.int8), ref.i8_codes(v[other])[0])
        else:
            assert same_codes(ref.unpack_act(q.cpu(), T, K)[other], ref.act_codes(v[other])[0])
            assert bool(((ref.unpack_act(q.cpu(), T, K)[[1, 3, 4]] & 0x7F) == 0x7F).any(dim=1).all())


@pytest.mark.parametrize("T,K", [(3, 400), (701, 400), (2100, 400)])
def test_norm_in_place_and_with_gaps_between_rows(T, K):
    x, r = ref.rows(1, T, K, F16), ref.rows(2, T, K, F16)
    weight = 1.0 + 0.1 * torch.randn(K, generator=torch.Generator().manual_seed(1))
    h, v = ref.norm(x, weight, EPS, r)
    xw, rw = torch.full((T, K + 16), 3.0, dtype=F16, device=DEV), torch.full((T, K + 8), 5.0, dtype=F16, device=DEV)
    xw[:, :K], rw[:, :K] = x.to(DEV), r.to(DEV)
    y, total, q, s = haq.haq_rmsnorm_quant(xw[:, :K], weight.to(DEV), EPS, haq.HAQ_CODES_I8, residual=rw[:, :K], sum_out=rw[:, :K], y=xw[:, :K])
    assert same_bits(rw[:, :K], h) and same_bits(xw[:, :K], v.to(F16))
    assert bool((xw[:, K:] == 3.0).all()) and bool((rw[:, K:] == 5.0).all())
    R = ref.padded_rows(T)
    for codes, dt, n in ((haq.HAQ_CODES_I8, torch.int8, T + 4), (haq.HAQ_CODES_E4M3, torch.float8_e4m3fn, 4 * R)):
        q = torch.full((448 * R,), 0x55, dtype=torch.uint8, device=DEV)
        s = torch.full((n,), -7.0, device=DEV)
        check_norm(x, weight, r, codes, False, q_packed=q.view(dt), scale=s)
        assert bool((q.view(-1, R, 16)[:, T:] == 0x55).all()) and bool((q.view(-1, R, 16)[K // 16:] == 0x55).all())
        assert bool((s[T:] == -7.0).all()) if codes == haq.HAQ_CODES_I8 else bool((s.view(4, R)[:, T:] == -7.0).all())


# ---- together -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T", [1, 37, 300])
def test_a_layer_of_them(T):
    """norm -> e4m3 linear -> norm with the residual -> int8 linear, on another stream, and captured in a graph: every replay equals
    the eager run on what its inputs hold then."""
    K, N = 512, 528
    wq, sw, wp, swd = weights(2, K, K)
    w2 = (torch.randn(K, N, generator=torch.Generator().manual_seed(4)) * 0.02).to(DEV)
    w2q, sw2 = haq.haq_quant_weight(w2, None)
    w2p = haq.haq_pack_weight(w2q)
    g1 = torch.ones(K, device=DEV)
    x = ref.rows(1, T, K, F16).to(DEV)
    bufs = {}

    def layer():
        _, _, q, s = haq.haq_rmsnorm_quant(x, g1, EPS, haq.HAQ_CODES_E4M3)
        a = haq.haq_gemm_fp8_packed(q, s, wp, swd, T, K, K)
        _, h, q8, s8 = haq.haq_rmsnorm_quant(a, g1, EPS, haq.HAQ_CODES_I8, residual=x)
        bufs.update(h=h, a=a, y=haq.haq_gemm_w8a8_packed(q8, s8, w2p, sw2, T, K, N), b=haq.haq_fp8_linear(x, wp, swd, K))
        return bufs["y"]

    want = layer().clone()
    h, v = ref.norm(x.cpu(), g1.cpu(), EPS)
    ref.assert_linear(bufs["a"].cpu(), *ref.linear(*ref.act_codes(v), wq, sw))
    q8, s8 = ref.i8_codes(ref.norm(bufs["a"].cpu(), g1.cpu(), EPS, x.cpu())[1])
    y = (q8.double() @ w2q.cpu().double()) * s8.double()[:, None] * sw2.cpu().double()
    # three roundings of binary32 and one of binary16
    assert bool(((want.cpu().double() - y).abs() <= y.abs() * (2.0 ** -11 + 2.0 ** -22) + 2.0 ** -25).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = layer()
        again_b = bufs["b"]
    side.synchronize()
    assert same_bits(again, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer()
    out_b = bufs["b"]
    for k in range(3):
        x.copy_(ref.rows(10 + k, T, K, F16))
        graph.replay()
        got, got_b = out.clone(), out_b.clone()
        torch.cuda.synchronize()
        assert same_bits(layer(), got) and same_bits(bufs["b"], got_b)


def test_norm_feeds_the_routed_experts():
    """16-bit rows of the norm into the expert FFN: the same bits as from rows computed apart."""
    from tests import offline
    from tests.gpu_util import dev, upload_experts
    m = offline.small_moe(seed=6, T=40, H=128, I=320, E=8)
    x = dev(m["X"])
    g = torch.ones(128, device=DEV)
    y, _, _, _ = haq.haq_rmsnorm_quant(x, g, EPS)
    _, v = ref.norm(x.cpu(), g.cpu(), EPS)
    experts = upload_experts(m["experts"])
    a = haq.haq_moe_w8a8_ffn(y, dev(m["logits"]), dev(m["s_in"]), experts, 320)
    b = haq.haq_moe_w8a8_ffn(v.to(F16).to(DEV), dev(m["logits"]), dev(m["s_in"]), experts, 320)
    assert same_bits(a, b)
