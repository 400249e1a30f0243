"""The step that README.md shows runs as it is written there, with the densify calls' workspace bound before it, and its gradients are right."""
import os
import textwrap

import numpy as np
import pytest
import torch

import oracle
from oracle import operators as op
from paper_1905_04035_amd import binding as ts
from paper_1905_04035_amd import workloads as wl
from tests.parity import DEV, TOL

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def example():
    """The indented lines behind the paragraph that begins with "From Python"."""
    with open(README) as f:
        lines = f.read().split("From Python", 1)[1].split("\n")
    first = next(i for i, l in enumerate(lines) if l.startswith("    "))
    last = next(i for i in range(first, len(lines)) if lines[i] and not lines[i].startswith("    "))
    return textwrap.dedent("\n".join(lines[first:last]))


def test_the_example_is_python():
    compile(example(), "README.md", "exec")


@pytest.mark.gpu
def test_the_example_runs_and_its_gradients():
    n, d, V = 1021, 128, 1777
    assert ts.ts_matmul_workspace_bytes(V, d, n) > ts.ts_workspace_bytes(n, d, V)          # dW is split along the tokens
    g = torch.Generator().manual_seed(1)
    E4M3, E5M2 = ts.TS_FP8_E4M3, ts.TS_FP8_E5M2
    names = dict(torch=torch, n=n, d=d, V=V, seed=11, offset=12,
                 ids=torch.randint(-1, V, (n,), generator=g, dtype=torch.int32).to(DEV), weight=(torch.randn(V, d, generator=g) * d ** -0.5).to(DEV),
                 pos=torch.randn(64, d, generator=g).to(DEV), pos_ids=(torch.arange(n) % 64).to(torch.int32).to(DEV),
                 dlogits=(torch.randn(n, V, generator=g) * 0.01).to(DEV), dtokens=(torch.randn(n, d, generator=g) * 0.01).to(DEV),
                 hidden=torch.empty(n, d, device=DEV), logits=torch.empty(n, V, dtype=torch.bfloat16, device=DEV),
                 dhidden=torch.empty(n, d, device=DEV), dweight=torch.empty(V, d, device=DEV),
                 h=ts.fp8_empty(n, d, E4M3), h_turned=ts.fp8_empty(d, n, E4M3), w=ts.fp8_empty(V, d, E4M3), w_turned=ts.fp8_empty(d, V, E4M3),
                 dl=ts.fp8_empty(n, V, E5M2), dl_turned=ts.fp8_empty(V, n, E5M2))
    ws = ts.Workspace(n, d, V)                                        # what the densify calls alone need
    try:
        exec(example(), names)
        torch.cuda.synchronize()
    finally:
        ts.ts_bind_workspace(None)
        del ws

    def product(a, fa, b):
        pair = [(q.view(torch.uint8).cpu().numpy(), s.cpu().numpy()) for q, s in (names[a], names[b])]
        return op.matmul(*pair[0], fa, *pair[1], E4M3)

    logits, size = product("h", E4M3, "w")
    got = names["logits"].double().cpu().numpy()
    # K sums, cut at 2^-23 each at most; a bf16 result's products at 7 * 2^-13 of their groups, and rounded at 2^-8
    assert (np.abs(got - logits) <= ((d + 1) * 2.0 ** -23 + 7 * 2.0 ** -13) * size * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(logits)).all()
    dhidden, size = product("dl", E5M2, "w_turned")
    assert (np.abs(names["dhidden"].double().cpu().numpy() - dhidden) <= (V + 1) * 2.0 ** -23 * size).all()
    dweight, size = product("dl_turned", E5M2, "h_turned")
    ids, dtokens = names["ids"].cpu().numpy(), names["dtokens"].cpu().numpy()
    rows = np.where(op.kept(n, d, 0.1, 11, 12), dtokens * np.float32(op.factor(0.1, d ** 0.5)), np.float32(0.0)).astype(np.float32)
    r = oracle.densify([ids], [rows], d, V, np.zeros((V, d), np.float32), wl.ROW_FP32)
    # the product's error, then that of the lookups' sums onto it (their magnitudes and the product's)
    bound = (n + 1) * 2.0 ** -23 * size + TOL * (r.abs_sum + size)
    assert (np.abs(names["dweight"].double().cpu().numpy() - dweight - r.exact) <= bound).all()
