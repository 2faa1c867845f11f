"""The weight gradient of 8-bit rows with offsets that are not in order or point outside the rows: a group's is the sum over the rows that its own two offsets name, whether or not they lie
behind the first offset.  Bounds as in test_gpu_gated.py."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2603_05500_amd as px
from tests.test_gpu_gated import U24, host, mx8_of, mx8_values, scratch, split_mx8
from tests.test_gpu_grouped import CODE, DT
from tests.test_gpu_grouped_offsets import KINDS, disorder

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("groups,rows,m,n", [(4, 100, 128, 128), (5, 1000, 130, 258), (8, 3000, 520, 1032), (3, 4000, 257, 263), (64, 4000, 256, 320), (300, 2000, 64, 136), (2, 8000, 129, 130)])
def test_weight_gradient_of_mx8_rows(lib, groups, rows, m, n, dtype, kind):
    """Rows that no group's own offsets name hold NaN, and so does the scratch."""
    offsets = disorder(kind, groups, rows)
    at = np.clip(offsets, 0, rows)
    named = np.zeros(rows, bool)
    for p, q in zip(at, at[1:]):
        named[p:q] = True
    rng, dt = np.random.default_rng(m + n), DT[dtype]
    x, z = (np.where(named[:, None], rng.standard_normal((rows, d)), np.nan) for d in (m, n))
    dZ = torch.from_numpy(z * 0.1).to(dt).cuda()
    Q = mx8_of(torch.from_numpy(x).to(dt).cuda())
    xh, zh = mx8_values(*split_mx8(Q, rows, m), m), host(dZ).numpy()
    desc = px.make_grouped_desc(m, n, groups, rows, CODE[dtype], px.GROUPED_X_MX8)
    flat = torch.full((groups * n * m + 64,), 3.0, device="cuda")
    dW = flat[: groups * n * m].view(groups, n, m)
    px.poetx_grouped_bwd_weight(desc, Q, dZ, torch.from_numpy(offsets.astype(np.int32)).cuda(), dW, False, scratch(px.poetx_grouped_workspace_bytes(desc)))
    got = host(dW).numpy()
    for g in range(groups):
        p, q = at[g], max(at[g], at[g + 1])
        ref, mag = zh[p:q].T @ xh[p:q], np.abs(zh[p:q]).T @ np.abs(xh[p:q])
        assert (np.abs(got[g] - ref) <= (q - p + 4) * U24 * mag + 2 * U24 * np.abs(ref) + 1e-37).all(), g
    assert bool((flat[groups * n * m:] == 3.0).all())
