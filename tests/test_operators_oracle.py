"""What pins the oracle of dropout, lookup and 8-bit products (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import operators as op


def test_philox_known_answers():
    # the published known answers of Philox4x32 for an all-zero and an all-one counter and key (ten and seven rounds)
    ones = 0xFFFFFFFF
    for rounds, counter, key, want in (
            (10, (0,) * 4, (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            (10, (ones,) * 4, (ones, ones), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            (7, (0,) * 4, (0, 0), (0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48))):
        assert tuple(int(x) for x in op.philox(counter, key, rounds)) == want


@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_share_of_kept_elements(p):
    # n independent draws: five standard deviations
    n = 400000
    keep = op.kept(100, n // 100, p, 0x123456789ABCDEF, 7)
    assert abs(keep.mean() - (1 - p)) < 5 * np.sqrt(p * (1 - p) / n)
    for other in (op.kept(100, n // 100, p, 0x123456789ABCDEF, 8), op.kept(100, n // 100, p, 0x123456789ABCDEE, 7)):
        agree = p * p + (1 - p) * (1 - p)
        assert abs((keep == other).mean() - agree) < 5 * np.sqrt(agree * (1 - agree) / n)


def test_a_mask_goes_by_the_element_s_place():
    whole = op.kept(40, 12, 0.5, 5, 6)
    assert np.array_equal(op.kept(10, 12, 0.5, 5, 6, first_row=30), whole[30:])
    assert np.array_equal(op.kept(20, 24, 0.5, 5, 6).ravel(), whole.ravel())
    assert np.array_equal(op.kept(4, 4, 0.0, 5, 6), np.ones((4, 4), bool))
    far = op.kept(1, 8, 0.5, 5, 6, first_row=1 << 40)            # beyond 2^32 groups of four
    assert far.shape == (1, 8) and not np.array_equal(op.kept(64, 8, 0.5, 5, 6, first_row=1 << 31), op.kept(64, 8, 0.5, 5, 6))


def test_gradient_of_the_lookup_is_the_dropped_densify():
    rng = np.random.default_rng(3)
    V, d, n, p, scale = 9, 8, 30, 0.3, 2.5
    ids = rng.integers(-1, V + 1, n)
    w, g = rng.standard_normal((V, d)), rng.standard_normal((n, d))
    rows = op.dropout(g, p, 1, 2, scale=scale)
    grad = np.zeros((V, d))
    ok = (ids >= 0) & (ids < V)
    np.add.at(grad, ids[ok], rows[ok])
    loss = lambda w: float((op.lookup(ids, w, scale, p, 1, 2) * g).sum())
    for v, j in ((0, 0), (3, 5), (8, 7)):
        step = np.zeros((V, d))
        step[v, j] = 0.5                                          # linear in w: a wide step loses nothing
        # factor() is rounded to 32 bits once with and once without the scale
        assert abs(loss(w + step) - loss(w - step) - grad[v, j]) < 1e-6 * (1 + np.abs(rows[ids == v]).sum())


@pytest.mark.parametrize("fmt,dtype", [(0, torch.float8_e4m3fn), (1, torch.float8_e5m2)])
def test_codes_against_another_encoder(fmt, dtype):
    v = op.decode(fmt)
    assert np.array_equal(torch.arange(256, dtype=torch.uint8).view(dtype).double().numpy(), v, equal_nan=True)
    top = op.FORMATS[fmt][2]
    grid = v[:int(np.flatnonzero(v == top)[0]) + 1]
    rng = np.random.default_rng(fmt)
    x = rng.standard_normal(20000) * 10.0 ** rng.uniform(-7, 2, 20000)
    x = np.concatenate([x, (grid[1:] + grid[:-1]) / 2, -(grid[1:] + grid[:-1]) / 2, grid, [0.0, -0.0]]).astype(np.float32)
    x = x[np.abs(x) <= top]
    assert np.array_equal(op.encode(x, fmt), torch.from_numpy(x).to(dtype).view(torch.uint8).numpy())


@pytest.mark.parametrize("fmt", [0, 1])
def test_scales(fmt):
    top = op.FORMATS[fmt][2]
    # exactly at the largest value, a step above it, a power of two, zero, the smallest and the largest numbers
    most = np.array([top, np.nextafter(np.float32(top), np.float32(np.inf)), 1.0, 0.0, 2.0 ** -149, 3.4028234e38, top / 4, top * 2.0 ** -60])
    x = np.zeros((len(most), 130))
    x[:, 77] = -most
    x[:, 129] = 1.0
    codes, scales = op.quantize(x, fmt)
    back = op.values(codes, scales, fmt)
    e = scales[:, 0].astype(int) - 127
    assert (most <= top * np.ldexp(1.0, e)).all() and ((most > top * np.ldexp(1.0, e - 1)) | (e == -127)).all()
    assert e[0] == 0 and e[1] == 1 and e[3] == -127 and e[4] == -127
    assert np.array_equal(back[:, 129], np.ones(len(most))) and (codes[:, 130:] == 0).all() and (scales[:, 2:] == 0).all()
    bits = op.FORMATS[fmt][0]
    assert (np.abs(back[:, 77] + most) <= most * 2.0 ** (-bits - 1) + np.ldexp(1.0, e) * 2.0 ** -17).all()


def test_product():
    rng = np.random.default_rng(5)
    a, b = rng.integers(-8, 9, (3, 300)).astype(float), rng.integers(-8, 9, (5, 300)).astype(float)
    (qa, sa), (qb, sb) = op.quantize(a, 0), op.quantize(b, 1)
    assert np.array_equal(op.values(qa, sa, 0)[:, :300], a)        # whole numbers to 16: exact in e4m3
    b = op.values(qb, sb, 1)[:, :300]
    want = np.array([[sum(a[i, k] * b[j, k] for k in range(300)) for j in range(5)] for i in range(3)])
    y, size = op.matmul(qa, sa, 0, qb, sb, 1)
    assert np.array_equal(y, want) and np.array_equal(size, np.abs(a) @ np.abs(b).T)
