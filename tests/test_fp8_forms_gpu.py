"""Every form of the 8-bit products at sizes and with values that the first tests of them leave out: bf16 results of few rows exactly, blocks
whose scales lie close together, so that no block hides behind another, what is no number in tiles and parts, the longest contracted axis,
results wider than 2^20 onto a tensor, one operand twice, and the same bits again."""
import functools

import numpy as np
import pytest
import torch

from oracle import operators as op
from paper_1905_04035_amd import binding as ts
from tests.parity import DEV
from tests.test_fp8_gpu import BF16, E4M3, E5M2, FP32, PRODUCTS, bind, on_gpu, operand, product, quantized, same_codes

pytestmark = pytest.mark.gpu

K_MAX = (1 << 24) - 128


def rounded(x, dtype):
    return torch.from_numpy(x).to(dtype).double().numpy()


def bound(K, dtype, want, size):
    """K sums, each off by at most 2^-23 of a partial sum; a bf16 result's products are cut at 7 * 2^-13 of their groups, and it is rounded at 2^-8."""
    tol = (K + 1) * 2.0 ** -23 * size
    return tol if dtype == FP32 else (tol + 7 * 2.0 ** -13 * size) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)


@pytest.mark.parametrize("M,N,K", PRODUCTS)
@pytest.mark.parametrize("fa,fb", [(E4M3, E4M3), (E5M2, E4M3)])
def test_bf16_products_of_whole_numbers_are_rounded_once(M, N, K, fa, fb):
    a, sa = operand(M, K, fa, "whole", M + K)
    b, sb = operand(N, K, fb, "whole", N + K + 1)
    want, size = op.matmul(a, sa, fa, b, sb, fb)
    # products of 1 to 256 lie within the 13 bits that the 8-bit instructions keep of a group, and sums are whole numbers below 2^24
    assert size.max() < 2 ** 24 and np.array_equal(want, np.rint(want))
    assert np.array_equal(product(a, sa, fa, b, sb, fb, K, BF16), rounded(want, BF16))


def close_scales(rows, K, fmt, seed):
    """Codes of one size and scales within 2^-3 .. 2^3 of each other: each block is a fair share of every sum."""
    rng = np.random.default_rng(seed)
    blocks = -(-K // 128)
    codes = np.zeros((rows, blocks * 128), dtype=np.uint8)
    scales = np.zeros((rows, -(-blocks // 4) * 4), dtype=np.uint8)
    codes[:, :K] = op.encode(np.clip(rng.standard_normal((rows, K)) * 40, -400, 400), fmt)
    scales[:, :blocks] = rng.integers(114, 121, (rows, blocks))
    return codes, scales


@pytest.mark.parametrize("M,N,K", [s for s in PRODUCTS if s[0] * s[1] * s[2] < 3e8])
@pytest.mark.parametrize("fa,fb", [(E4M3, E4M3), (E5M2, E4M3), (E4M3, E5M2), (E5M2, E5M2)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_products_of_blocks_with_close_scales(M, N, K, fa, fb, dtype):
    (a, sa), (b, sb) = close_scales(M, K, fa, M + K), close_scales(N, K, fb, N + K + 1)
    want, size = op.matmul(a, sa, fa, b, sb, fb)
    assert (np.abs(product(a, sa, fa, b, sb, fb, K, dtype) - want) <= bound(K, dtype, want, size)).all()


# few rows with one, two and four wavefronts along K and both widths; every size of tile, whole and in parts
FORMS = [(3, 40, 300), (20, 36, 200), (9, 6008, 4100), (30, 6008, 1100), (100, 130, 520), (1239, 1024, 3419), (280, 181, 20000), (1280, 1920, 4000),
         (4000, 700, 1000), (2300, 4100, 700)]


@functools.lru_cache(maxsize=2)
def whole_numbers(M, N, K, fa):
    a, sa = operand(M, K, fa, "whole", 1)
    b, sb = operand(N, K, E4M3, "whole", 2)
    want, size = op.matmul(a, sa, fa, b, sb, E4M3)
    assert size.max() < 2 ** 24
    return a, sa, b, sb, want


@pytest.mark.parametrize("code", [0x7C, 0x7D, 0x7F, 0xFC, 0xFF])
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("fa", [E4M3, E5M2])
@pytest.mark.parametrize("M,N,K", FORMS)
def test_what_is_no_number_reaches_its_row_and_column_alone(M, N, K, fa, dtype, code):
    if np.isfinite(op.decode(fa)[code]):
        code = 0x7F
    a, sa, b, sb, want = (x.copy() for x in whole_numbers(M, N, K, fa))
    i, j = M * 2 // 3, N // 3
    a[i, K - 1] = code                                               # in the last block, and in one of the first
    b[j, min(K - 1, 130)] = 0x7F
    got = product(a, sa, fa, b, sb, E4M3, K, dtype)
    assert not np.isfinite(got[i]).any() and np.isnan(got[:, j]).all()
    rest = np.ones((M, N), bool)
    rest[i], rest[:, j] = False, False
    assert np.array_equal(got[rest], rounded(want, dtype)[rest])


@pytest.mark.parametrize("M,N", [(20, 48), (70, 40), (512, 512), (600, 520)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_the_longest_contracted_axis(M, N, dtype):
    """Whole numbers at a few places of it, its ends and the ends of blocks among them; zeros elsewhere."""
    K, rng = K_MAX, np.random.default_rng(M)
    at = np.unique(np.concatenate([[0, 1, 127, 128, K // 2 - 1, K // 2, K - 129, K - 128, K - 1], rng.integers(0, K, 40)]))
    ops, values = [], []
    for rows in (M, N):
        q, s = ts.fp8_empty(rows, K, E4M3)
        v = rng.integers(-4, 5, (rows, len(at)))
        q.view(torch.uint8).zero_()
        q.view(torch.uint8)[:, torch.from_numpy(at).to(DEV)] = torch.from_numpy(op.encode(v, E4M3)).to(DEV)
        s.fill_(127)
        ops += [q, s]
        values.append(v.astype(np.float64))
    out = torch.full((M, N), float("nan"), dtype=dtype, device=DEV)
    ws = bind(M, N, K)
    try:
        ts.ts_matmul_fp8(*ops, K, out)
        torch.cuda.synchronize()
    finally:
        ts.ts_bind_workspace(None)
        del ws
    assert np.array_equal(out.double().cpu().numpy(), rounded(values[0] @ values[1].T, dtype))
    del ops
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M,N,K", [(70, 1100000, 100), (300, 1048580, 130), (5, 1100001, 64)])
@pytest.mark.parametrize("in_place", [False, True])
def test_onto_a_tensor_of_more_than_2_to_the_20_columns(M, N, K, in_place):
    a, sa = operand(M, K, E4M3, "whole", 1)
    few, sfew = operand(999, K, E5M2, "whole", 2)                    # rows that repeat
    times = -(-N // 999)
    b = on_gpu(np.tile(few, (times, 1))[:N], np.tile(sfew, (times, 1))[:N], E5M2)
    want = torch.from_numpy(op.values(a, sa, E4M3) @ op.values(few, sfew, E5M2).T).float().to(DEV).repeat(1, times)[:, :N]
    c_in = torch.randint(-1000, 1001, (M, N), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).float()
    want = want + c_in
    out = c_in if in_place else torch.full((M, N), float("nan"), device=DEV)
    ws = bind(M, N, K)
    try:
        ts.ts_matmul_fp8(*on_gpu(a, sa, E4M3), *b, K, out, c_in)
        torch.cuda.synchronize()
    finally:
        ts.ts_bind_workspace(None)
        del ws
    assert torch.equal(out, want)
    del want, c_in, out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M,K", [(7, 300), (200, 1000), (700, 20000), (3000, 260)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_one_operand_twice(M, K, dtype):
    a, sa = operand(M, K, E4M3, "whole", 5)
    u = on_gpu(a, sa, E4M3)
    out = torch.empty(M, M, dtype=dtype, device=DEV)
    ws = bind(M, M, K)
    try:
        ts.ts_matmul_fp8(*u, *u, K, out)
        torch.cuda.synchronize()
    finally:
        ts.ts_bind_workspace(None)
        del ws
    v = op.values(a, sa, E4M3)
    assert np.array_equal(out.double().cpu().numpy(), rounded(v @ v.T, dtype))


@pytest.mark.parametrize("M,N,K", [(8192, 32768, 1024), (8192, 8192, 2048), (5001, 33801, 1000), (8500, 2100, 5000), (33801, 1024, 4987), (300, 1024, 20000), (32, 32768, 1024)])
@pytest.mark.parametrize("kind", ["bf16", "fp32", "onto"])
def test_the_same_bits_again(M, N, K, kind):
    g = torch.Generator(device=DEV).manual_seed(M)
    pairs = []
    for rows in (M, N):
        pairs.append(ts.fp8_empty(rows, K))
        ts.ts_quantize_fp8(torch.randn(rows, K, generator=g, device=DEV), E4M3, *pairs[-1])
    c_in = torch.randn(M, N, generator=g, device=DEV) if kind == "onto" else None
    ws = bind(M, N, K)
    outs = [torch.full((M, N), float("nan"), dtype=BF16 if kind == "bf16" else FP32, device=DEV) for _ in range(2)]
    try:
        ts.ts_matmul_fp8(*pairs[0], *pairs[1], K, outs[0], c_in)
        for _ in range(5):
            ws.fill_(0xFF)
            outs[1].fill_(float("nan"))
            ts.ts_matmul_fp8(*pairs[0], *pairs[1], K, outs[1], c_in)
            torch.cuda.synchronize()
            assert torch.equal(*outs)
    finally:
        ts.ts_bind_workspace(None)
        del ws
    del outs, c_in, pairs
    torch.cuda.empty_cache()


@pytest.mark.parametrize("turned", [False, True])
def test_codes_of_the_longest_row_and_column(turned):
    """2^31 - 1 elements along the blocks' axis, a few of them no zeros."""
    n = (1 << 31) - 1
    x = torch.zeros((n, 1) if turned else (1, n), dtype=BF16, device=DEV)
    at = torch.tensor([0, 5, 127, 128, 1 << 30, (1 << 30) + 127, n - 1000, n - 2, n - 1], device=DEV)
    v = torch.tensor([1.0, -3.0, 448.0, 2.0 ** -9, 5.0, -6.0, 2.0 ** 40, 7.0, 0.3]).to(BF16)
    x.view(-1)[at] = v.to(DEV)
    q, s = ts.fp8_empty(1, n, E4M3)
    q.view(torch.uint8).fill_(0x55)
    s.fill_(0x55)
    ts.ts_quantize_fp8(x, E4M3, *((None, None, q, s) if turned else (q, s)))
    torch.cuda.synchronize()
    blocks = torch.unique(at // 128)
    for b in blocks.tolist():
        part = torch.zeros(128)
        end = min(n, (b + 1) * 128)
        part[:end - b * 128] = x.view(-1)[b * 128:end].float().cpu()
        want, want_scales = op.quantize(part[None].numpy(), E4M3)
        assert int(s[0, b]) == want_scales[0, 0]
        same_codes(q[:, b * 128:(b + 1) * 128], want, E4M3)
    assert int((s != 0).sum()) == len(blocks) and int(torch.count_nonzero(q.view(torch.uint8))) == len(at)
    del x, q, s
    torch.cuda.empty_cache()
