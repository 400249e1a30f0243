"""One training step around a shared embedding, as a program makes it, on one stream: tokens looked up and dropped, the projection
in 8 bits with the same weight, the gradients of the logits turned into that of the hidden states and that of the weight, and the lookups'
gradients added to it.  Against the same step in float64 on the CPU, with the codes and scales that the GPU made (these are compared
bit for bit elsewhere)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import operators as op
from paper_1905_04035_amd import binding as ts
from paper_1905_04035_amd import workloads as wl
from tests.parity import DEV, TOL

pytestmark = pytest.mark.gpu


def quantized(x, fmt, ways):
    """(codes, scales) of x and, if asked for, of its transpose; on the GPU."""
    out = {}
    if "rows" in ways:
        out["rows"] = ts.fp8_empty(x.shape[0], x.shape[1], fmt)
    if "columns" in ways:
        out["columns"] = ts.fp8_empty(x.shape[1], x.shape[0], fmt)
    none = (None, None)
    ts.ts_quantize_fp8(x, fmt, *out.get("rows", none), *out.get("columns", none))
    return out


def product(a, b, fa, fb, K, out, c_in=None):
    """The call, and its result in float64."""
    ts.ts_matmul_fp8(*a, *b, K, out, c_in)
    host = [(q.view(torch.uint8).cpu().numpy(), s.cpu().numpy()) for q, s in (a, b)]
    return op.matmul(*host[0], fa, *host[1], fb, None if c_in is None else c_in.cpu().numpy())


@pytest.mark.parametrize("n,d,V", [(300, 64, 1000), (1021, 128, 1777)])
def test_a_step(n, d, V):
    gen = torch.Generator().manual_seed(n)
    weight = torch.randn(V, d, generator=gen).mul_(d ** -0.5).to(DEV)
    pos = torch.randn(64, d, generator=gen).to(DEV)
    ids = torch.randint(-1, V, (n,), generator=gen, dtype=torch.int32).to(DEV)            # some padding
    at = (torch.arange(n) % 64).to(torch.int32).to(DEV)
    upstream = (torch.randn(n, d, generator=gen) * 0.01).to(DEV)                          # of the tokens, from the network behind them
    dlogits = (torch.randn(n, V, generator=gen) * 0.01).to(torch.bfloat16).to(DEV)
    scale, mask = d ** 0.5, ts.DropoutMask(0.1, 1234, 5)
    need = max([ts.ts_workspace_bytes(n, d, V)] + [ts.ts_matmul_workspace_bytes(*s) for s in ((n, V, d), (n, d, V), (V, d, n))])
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    ts.ts_bind_workspace(ws)
    try:
        # forward: tokens, and (the network being the identity) logits
        hidden = torch.empty(n, d, device=DEV)
        ts.ts_lookup_dropout(ids, weight, scale, mask, hidden, pos, at)
        h, w = quantized(hidden, ts.TS_FP8_E4M3, ("rows", "columns")), quantized(weight, ts.TS_FP8_E4M3, ("rows", "columns"))
        logits = torch.empty(n, V, dtype=torch.bfloat16, device=DEV)
        want_logits, size_logits = product(h["rows"], w["rows"], 0, 0, d, logits)
        # backward: of the hidden states, and of the weight; then the lookups' share of it, in place
        g = quantized(dlogits, ts.TS_FP8_E5M2, ("rows", "columns"))
        dhidden, dweight = torch.empty(n, d, device=DEV), torch.empty(V, d, device=DEV)
        want_dhidden, size_dhidden = product(g["rows"], w["columns"], 1, 0, V, dhidden)
        want_dense, size_dense = product(g["columns"], h["columns"], 1, 0, n, dweight)
        dense = dweight.clone()
        ts.ts_densify_dropout(ids, upstream, d, V, scale, mask, dweight, dweight)
        torch.cuda.synchronize()
    finally:
        ts.ts_bind_workspace(None)

    want_hidden = op.lookup(ids.cpu().numpy(), weight.cpu().numpy(), scale, 0.1, 1234, 5, pos.cpu().numpy(), at.cpu().numpy())
    assert (np.abs(hidden.cpu().numpy() - want_hidden) <= 2.02 * 2.0 ** -24 * np.abs(want_hidden)).all()          # two roundings
    # sums of K products, cut at 2^-23 each at most; the bf16 result's products at 7 * 2^-13 of their groups, and rounded at 2^-8
    cut = (d + 1) * 2.0 ** -23 + 7 * 2.0 ** -13
    assert (np.abs(logits.double().cpu().numpy() - want_logits) <= cut * size_logits * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want_logits)).all()
    assert (np.abs(dhidden.cpu().numpy() - want_dhidden) <= (V + 1) * 2.0 ** -23 * size_dhidden).all()
    assert (np.abs(dense.cpu().numpy() - want_dense) <= (n + 1) * 2.0 ** -23 * size_dense).all()
    # the whole gradient: the lookups' rows, rounded once, onto what the product left
    rows = (op.kept(n, d, 0.1, 1234, 5) * (upstream.cpu().numpy() * np.float32(op.factor(0.1, scale)))).astype(np.float32)
    r = oracle.densify([ids.cpu().numpy()], [rows], d, V, dense.cpu().numpy(), wl.ROW_FP32)
    assert (np.abs(dweight.cpu().numpy().astype(np.float64) - r.exact) <= TOL * r.abs_sum).all() and r.n_bad == int((ids < 0).sum())
    # and the codes cost what 3 and 2 mantissa bits cost: against the exact gradient of the exact logits' gradient, half a step of either factor
    exact = dlogits.double().cpu().numpy().T @ hidden.double().cpu().numpy()
    terms = np.abs(dlogits.double().cpu().numpy()).T @ np.abs(hidden.double().cpu().numpy())
    # (below the smallest normal code a step is absolute: 2^-10 and 2^-17 of a block's scale, which is at most 2^-7 and 2^-14 of its largest)
    h_most, g_most = np.abs(hidden.cpu().numpy()).max(), np.abs(dlogits.float().cpu().numpy()).max()
    small = n * (h_most * 2.0 ** -17 * g_most + g_most * 2.0 ** -31 * h_most)
    assert (np.abs(dense.cpu().numpy() - exact) <= (2.0 ** -4 + 2.0 ** -3 + 2.0 ** -7 + 1e-3) * terms + small * 2).all()
