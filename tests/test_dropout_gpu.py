"""Dropout with a mask that is never stored, the lookup in front of it and the densify behind it, on the GPU against the
oracle.  Tolerances count roundings: half a step is 2^-24 (fp32) or 2^-8 (bf16) of the value."""
import numpy as np
import pytest
import torch

import oracle
from oracle import operators as op
from paper_1905_04035_amd import binding as ts
from paper_1905_04035_amd import workloads as wl
from tests.parity import DEV, TOL, error_bound

pytestmark = pytest.mark.gpu

FP32, BF16 = torch.float32, torch.bfloat16
SEED, OFFSET = 0x9E3779B97F4A7C15, (7 << 32) + 11
STEP = {FP32: 2.0 ** -24, BF16: 2.0 ** -8}


def values(shape, dtype, seed=1):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def near(got, want, dtype, roundings):
    """Every element within `roundings` fp32 roundings, and one to its type, of its own size; what is no number as it is."""
    got = host(got)
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)) and np.array_equal(got[~fine], want[~fine], equal_nan=True)
    got, want = got[fine], want[fine]
    bound = (roundings * STEP[FP32] + (STEP[BF16] if dtype == BF16 else 0.0)) * 1.01 * np.abs(want) + 2.0 ** -149
    assert (np.abs(got - want) <= bound).all(), float(np.max(np.abs(got - want) / np.maximum(bound, 1e-300)))


SHAPES = [(1, 4), (3, 4), (1, 12), (5, 20), (257, 64), (33, 516), (7, 1028), (2, 4100), (1000, 1024)]


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.75])
def test_dropout(n, d, dtype, p):
    x, add = values((n, d), dtype), values((n, d), dtype, 2)
    m = ts.DropoutMask(p, SEED, OFFSET)
    for residual in (None, add):
        out = torch.full((n, d), float("nan"), dtype=dtype, device=DEV)
        ts.ts_dropout(x.to(DEV), m, out, None if residual is None else residual.to(DEV))
        # one product and sum, rounded once (of a bf16 result: and once more)
        near(out, op.dropout(host(x), p, SEED, OFFSET, None if residual is None else host(residual)), dtype, 1)
        if residual is None:
            gone = ~op.kept(n, d, p, SEED, OFFSET)
            bits = out.cpu().view(torch.int32 if dtype == FP32 else torch.int16).numpy()
            assert (bits[gone] == 0).all()                            # +0.0, not -0.0


def test_dropout_of_what_is_no_number():
    n, d = 16, 64
    x = values((n, d), FP32)
    x.view(-1)[::3] = torch.tensor([float("nan"), float("inf"), float("-inf")]).repeat(n * d)[:len(x.view(-1)[::3])]
    out = torch.empty(n, d, device=DEV)
    ts.ts_dropout(x.to(DEV), ts.DropoutMask(0.5, 3, 4), out)
    keep = op.kept(n, d, 0.5, 3, 4)
    near(out, np.where(keep, host(x) * 2.0, 0.0), FP32, 1)


@pytest.mark.parametrize("place", ["x", "add"])
def test_dropout_in_place_and_its_neighbours(place):
    n, d = 37, 20
    x, add = values((n, d), BF16), values((n, d), BF16, 2)
    whole = torch.full((n + 8, d), 5.0, dtype=BF16, device=DEV)      # 16-byte aligned rows: 4 rows are 160 bytes
    inside = whole[4:4 + n]
    inside.copy_(x if place == "x" else add)
    other = (add if place == "x" else x).to(DEV)
    a, b = (inside, other) if place == "x" else (other, inside)
    ts.ts_dropout(a, ts.DropoutMask(0.2, 1), inside, b)
    near(inside, op.dropout(host(x), 0.2, 1, 0, host(add)), BF16, 1)
    assert (whole[:4] == 5).all() and (whole[4 + n:] == 5).all()


def test_backward_of_dropout_is_the_same_call():
    n, d = 19, 24
    m = ts.DropoutMask(0.3, 77, 5)
    x, g = values((n, d), FP32).to(DEV), values((n, d), FP32, 2).to(DEV)
    out, grad = torch.empty_like(x), torch.empty_like(x)
    ts.ts_dropout(x, m, out)
    ts.ts_dropout(g, m, grad)
    # a linear map that equals its transpose: <dropout(x), g> = <x, dropout(g)>, term by term to two roundings
    left, right = host(out) * host(g), host(x) * host(grad)
    assert (np.abs(left - right) <= 2.1 * 2.0 ** -24 * np.abs(left)).all() and (left != 0).any()


@pytest.mark.parametrize("n", [0, 1, 65])
@pytest.mark.parametrize("d", [4, 64, 68, 256, 260, 1024, 2052])
@pytest.mark.parametrize("wt,ot", [(FP32, FP32), (FP32, BF16), (BF16, BF16), (BF16, FP32)])
def test_lookup(n, d, wt, ot):
    V, P = 50, 9
    g = torch.Generator().manual_seed(n + d)
    ids = torch.randint(-2, V + 2, (n,), generator=g, dtype=torch.int32)        # some outside the vocabulary
    at = torch.randint(-1, P + 1, (n,), generator=g, dtype=torch.int32)
    w, pos = values((V, d), wt, 3), values((P, d), wt, 4)
    for with_pos, p in ((True, 0.1), (False, 0.1), (True, 0.0)):
        out = torch.full((n, d), float("nan"), dtype=ot, device=DEV)
        more = (pos.to(DEV), at.to(DEV)) if with_pos else ()
        ts.ts_lookup_dropout(ids.to(DEV), w.to(DEV), 3.3, ts.DropoutMask(p, SEED, OFFSET), out, *more)
        want = op.lookup(ids.numpy(), host(w), 3.3, p, SEED, OFFSET, *((host(pos), at.numpy()) if with_pos else ()))
        near(out, want, ot, 2)                                        # scale and position in one rounding, 1 / (1 - p) in one


def test_lookup_without_positions_in_the_table():
    out = torch.empty(3, 8, device=DEV)
    w = torch.ones(2, 8, device=DEV)
    ids = torch.tensor([0, 1, 7], dtype=torch.int32, device=DEV)
    ts.ts_lookup_dropout(ids, w, 2.0, ts.DropoutMask(0.0, 0), out, torch.empty(0, 8, device=DEV), ids)
    assert out.cpu().tolist() == [[2.0] * 8, [2.0] * 8, [0.0] * 8]


# shapes that take each form of the row reduction (one launch; pieces of 8, 16, 32; rows row by row) and rows of odd widths
DENSIFY = [(1, 4, 3), (2048, 64, 1000), (300, 12, 40), (3000, 100, 5000), (9000, 512, 3000), (16384, 256, 33801), (5000, 1028, 2000),
           (60000, 512, 8000), (100000, 256, 900), (70000, 1024, 500), (0, 8, 5)]


def pairs(n, d, V, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    ids = ((V ** torch.rand(n, generator=g, dtype=torch.float64)).long() - 1 + 3).remainder(V + 1).sub(1).to(torch.int32)      # -1 too
    return ids, torch.randn(n, d, generator=g).to(dtype), torch.randn(V, d, generator=g)


@pytest.mark.parametrize("n,d,V", DENSIFY)
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("in_place", [False, True])
def test_densify(n, d, V, dtype, in_place):
    ids, rows, dense = pairs(n, d, V, dtype)
    m, scale = ts.DropoutMask(0.25, SEED, OFFSET), 4.5
    ws = ts.Workspace(max(n, 1), d, V)
    try:
        dn = dense.to(DEV)
        out = dn if in_place else torch.full((V, d), float("nan"), device=DEV)
        ts.ts_densify_dropout(ids.to(DEV), rows.to(DEV), d, V, scale, m, dn, out)
        torch.cuda.synchronize()
        piece = ts.ts_last_launch_info()["piece_tokens"]
        # the value rows as the kernel makes them, rounded once to fp32
        f = np.float32(op.factor(0.25, scale))
        made = np.where(op.kept(n, d, 0.25, SEED, OFFSET), rows.float().numpy() * f, np.float32(0.0)).astype(np.float32)
        r = oracle.densify([ids.numpy()], [made], d, V, dense.numpy(), wl.ROW_FP32)
        got = out.cpu().numpy()
        none = r.count == 0
        assert np.array_equal(got[none].view(np.uint32), dense.numpy()[none].view(np.uint32))
        bound = min(TOL, 1.01 * error_bound(int(r.count.max(initial=0)), piece)) * r.abs_sum + 2.0 ** -149
        assert (np.abs(got.astype(np.float64) - r.exact) <= bound).all()
        if dtype == FP32 and n:                                       # ts_densify on those rows: the same bits
            again = torch.empty(V, d, device=DEV)
            ts.ts_densify(ids.to(DEV), torch.from_numpy(made).to(DEV), d, V, dense.to(DEV), again)
            assert torch.equal(again.view(torch.int32), out.view(torch.int32))
    finally:
        ws.close()


@pytest.mark.parametrize("n,d,V", [(2048, 64, 1000), (9000, 512, 3000), (60000, 1024, 8000)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_densify_without_dropout_is_densify(n, d, V, dtype):
    ids, rows, dense = (t.to(DEV) for t in pairs(n, d, V, dtype))
    ws = ts.Workspace(n, d, V)
    try:
        a, b = torch.empty_like(dense), torch.empty_like(dense)
        (ts.ts_densify if dtype == FP32 else ts.ts_densify_bf16)(ids, rows, d, V, dense, a)
        ts.ts_densify_dropout(ids, rows, d, V, 1.0, ts.DropoutMask(0.0, 1), dense, b)
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))
        ts.ts_densify_dropout(ids, rows, d, V, 1.0, ts.DropoutMask(0.0, 1), None, b)
        (ts.ts_densify if dtype == FP32 else ts.ts_densify_bf16)(ids, rows, d, V, None, a)
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))
    finally:
        ws.close()


def test_densify_drops_what_is_no_number():
    n, d, V = 200, 32, 10
    ids, rows, dense = pairs(n, d, V, FP32)
    keep = op.kept(n, d, 0.5, 9, 0)
    rows[torch.from_numpy(~keep)] = float("nan")                      # only dropped elements
    ws = ts.Workspace(n, d, V)
    try:
        out = torch.empty(V, d, device=DEV)
        ts.ts_densify_dropout(ids.to(DEV), rows.to(DEV), d, V, 1.0, ts.DropoutMask(0.5, 9), dense.to(DEV), out)
        assert torch.isfinite(out).all()
    finally:
        ws.close()


def test_gradients_against_differences():
    """Loss <lookup(W, P), g>: linear in the weight and the positions, so differences of any width are exact to rounding."""
    n, d, V, P, p, scale = 60, 8, 12, 7, 0.3, 2.0
    gen = torch.Generator().manual_seed(4)
    ids = torch.randint(0, V, (n,), generator=gen, dtype=torch.int32).to(DEV)
    at = torch.randint(0, P, (n,), generator=gen, dtype=torch.int32).to(DEV)
    w, pos, g = (torch.randint(-8, 9, s, generator=gen).float().to(DEV) for s in ((V, d), (P, d), (n, d)))
    m = ts.DropoutMask(p, 21, 3)

    def loss(w, pos):
        out = torch.empty(n, d, device=DEV)
        ts.ts_lookup_dropout(ids, w, scale, m, out, pos, at)
        return float((out.double() * g.double()).sum())

    ws = ts.Workspace(n, d, max(V, P))
    try:
        dw, dpos = torch.empty_like(w), torch.empty_like(pos)
        ts.ts_densify_dropout(ids, g, d, V, scale, m, None, dw)
        ts.ts_densify_dropout(at, g, d, P, 1.0, m, None, dpos)
    finally:
        ws.close()
    # n terms of at most 8 * (8 * 2 + 8) / 0.7 in size, two roundings each, in each of the two losses; the gradient's n terms likewise
    tol = 2.5 * 2.0 ** -24 * n * 8 * 30 / 0.7
    for grad, which in ((dw, 0), (dpos, 1)):
        for i, j in ((0, 0), (3, 5), (6, 7)):
            up, down = [w.clone(), pos.clone()], [w.clone(), pos.clone()]
            up[which][i, j] += 1.0
            down[which][i, j] -= 1.0
            assert abs((loss(*up) - loss(*down)) / 2 - float(grad[i, j])) <= tol


def test_a_mask_that_a_captured_graph_moves_on():
    n, d, V = 500, 64, 40
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    m = ts.DropoutMask(0.4, SEED, 1000, step)
    ids, rows, dense = (t.to(DEV) for t in pairs(n, d, V, FP32))
    ids = ids.clamp_min(0)
    w = torch.randn(V, d, generator=torch.Generator().manual_seed(8)).to(DEV)
    out, act, grad = torch.empty(n, d, device=DEV), torch.empty(n, d, device=DEV), torch.empty(V, d, device=DEV)
    ws = ts.Workspace(n, d, V)
    try:
        def work():
            ts.ts_lookup_dropout(ids, w, 1.5, m, out)
            ts.ts_dropout(rows, m, act, out)
            ts.ts_densify_dropout(ids, rows, d, V, 1.5, m, dense, grad)

        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            work()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            work()
        seen = []
        for k in range(4):
            step.fill_(k % 3)
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (out, act, grad)]
            eager = ts.DropoutMask(0.4, SEED, 1000 + k % 3)
            want = [torch.empty_like(t) for t in got]
            ts.ts_lookup_dropout(ids, w, 1.5, eager, want[0])
            ts.ts_dropout(rows, eager, want[1], want[0])
            ts.ts_densify_dropout(ids, rows, d, V, 1.5, eager, dense, want[2])
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            seen.append(got[0])
        assert not torch.equal(seen[0], seen[1]) and torch.equal(seen[0], seen[3])
    finally:
        ws.close()


def test_offsets_wrap_at_64_bits():
    n, d = 8, 16
    x = values((n, d), FP32).to(DEV)
    step = torch.full((1,), 5, dtype=torch.int64, device=DEV)
    out = torch.empty_like(x)
    ts.ts_dropout(x, ts.DropoutMask(0.5, (1 << 64) - 1, (1 << 64) - 2, step), out)
    near(out, op.dropout(host(x), 0.5, (1 << 64) - 1, 3), FP32, 1)


def test_streams_and_shapes_of_the_binding():
    n, d = 8, 16
    x, m = values((n, d), FP32).to(DEV), ts.DropoutMask(0.5, 1)
    s = torch.cuda.Stream()
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    ts.ts_dropout(x, m, out, stream=s)
    s.synchronize()
    near(out, op.dropout(host(x), 0.5, 1, 0), FP32, 1)
    ids = torch.zeros(n, dtype=torch.int32, device=DEV)
    for call in (lambda: ts.ts_dropout(x, m, out[:4]), lambda: ts.ts_dropout(x.t(), m, out), lambda: ts.ts_dropout(x, m, out.bfloat16()),
                 lambda: ts.ts_dropout(x.half(), m, out.half()), lambda: ts.ts_dropout(x, m, out, x[:4]),
                 lambda: ts.ts_dropout(x, ts.DropoutMask(0.5, 1, 0, torch.zeros(2, dtype=torch.int64, device=DEV)), out),
                 lambda: ts.ts_dropout(x, ts.DropoutMask(0.5, 1, 0, torch.zeros(1, dtype=torch.int64)), out),
                 lambda: ts.ts_lookup_dropout(ids[:4], x, 1.0, m, out), lambda: ts.ts_lookup_dropout(ids.long(), x, 1.0, m, out),
                 lambda: ts.ts_lookup_dropout(ids, x, 1.0, m, out, x), lambda: ts.ts_lookup_dropout(ids, x, 1.0, m, out, x.bfloat16(), ids),
                 lambda: ts.ts_densify_dropout(ids, x, d, n + 1, 1.0, m, x, out), lambda: ts.ts_densify_dropout(ids, x[:4], d, n, 1.0, m, x, out)):
        with pytest.raises(AssertionError):
            call()
    for mask in (ts.DropoutMask(0.5, -1), ts.DropoutMask(0.5, 1 << 64), ts.DropoutMask(0.5, 0, -1)):
        with pytest.raises(OverflowError):
            ts.ts_dropout(x, mask, out)
    with pytest.raises(ts.TsError):
        ts.ts_dropout(x, ts.DropoutMask(1.0, 1), out)


def test_elements_beyond_2_to_the_34():
    """Groups of four beyond 2^32: the counter's second word."""
    d, rows = 1 << 20, (1 << 14) + 2
    x = torch.empty(rows, d, dtype=BF16, device=DEV)                  # 34 GB, of which the ends are looked at
    x[0].fill_(1.0)
    x[-2:].fill_(1.0)
    ts.ts_dropout(x, ts.DropoutMask(0.5, 9, 1), x)
    for first, part in ((0, x[:1]), (rows - 2, x[-2:])):
        assert np.array_equal(host(part) == 2.0, op.kept(part.shape[0], d, 0.5, 9, 1, first_row=first))
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,d,V,used", [(2048, 64, 1000, 2048), (20000, 260, 5000, 20000), (70000, 1024, 9000, 70000), ((1 << 22) + 100, 4096, 1000, 100)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_densify_dropout_is_densify_of_dropped_rows(n, d, V, used, dtype):
    """Bit for bit with a factor of two, which rounds nothing.  The last rows lie beyond 2^34 elements, the others are padding."""
    if dtype == FP32 and n > 1 << 20:
        n = n // 4 + 75
    rows = torch.empty(n, d, dtype=dtype, device=DEV)
    rows[n - used:] = torch.randn(used, d, generator=torch.Generator().manual_seed(n)).to(dtype).to(DEV)
    ids = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    ids[n - used:] = torch.randint(0, V, (used,), generator=torch.Generator().manual_seed(d), dtype=torch.int32).to(DEV)
    dense = values((V, d), FP32).to(DEV)
    got, want = torch.empty_like(dense), torch.empty_like(dense)
    ws = torch.empty(ts.ts_workspace_bytes(n, d, V), dtype=torch.uint8, device=DEV)
    m = ts.DropoutMask(0.5, SEED, OFFSET)
    ts.ts_bind_workspace(ws)
    try:
        ts.ts_densify_dropout(ids, rows, d, V, 1.0, m, dense, got)
        ts.ts_dropout(rows, m, rows)
        (ts.ts_densify_bf16 if dtype == BF16 else ts.ts_densify)(ids, rows, d, V, dense, want)
        torch.cuda.synchronize()
    finally:
        ts.ts_bind_workspace(None)
    assert torch.equal(got.view(torch.int32), want.view(torch.int32))
    assert not torch.equal(got, dense)
    del rows
    torch.cuda.empty_cache()


def test_lookup_beyond_2_to_the_32():
    """Rows of a weight, and of the result, behind 2^32 elements."""
    d, V = 4096, (1 << 20) + 40
    weight = torch.empty(V, d, dtype=BF16, device=DEV)
    weight[-40:] = values((40, d), BF16).to(DEV)
    n = (1 << 20) + 9
    ids = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    last = torch.arange(V - 20, V - 11, dtype=torch.int32)
    ids[-9:] = last.to(DEV)
    out = torch.empty(n, d, dtype=BF16, device=DEV)
    ts.ts_lookup_dropout(ids, weight, 2.0, ts.DropoutMask(0.25, SEED, OFFSET), out)
    keep = op.kept(9, d, 0.25, SEED, OFFSET, first_row=n - 9)
    near(out[-9:], np.where(keep, host(weight[-20:-11]) * 2.0 / 0.75, 0.0), BF16, 2)
    assert not bool(out[:-9].any())
    del weight, out
    torch.cuda.empty_cache()
