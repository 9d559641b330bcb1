"""GPU tests of every kernel of the log-probabilities and their gradients: sizes that between them take each form in each
direction, type and way of multiplying (which ones they take is held by tests/test_host_launches.py), odd in rows, ids and
columns, against 64 bits.  Bounds as in tests/test_gpu_vocab.py."""
import math

import numpy as np
import pytest
import torch

import paper_2602_00482_amd as dta

pytestmark = pytest.mark.gpu

U, UM = 2.0 ** -24, 2.0 ** -23
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
KIND = {"bf16": dta.BF16, "f32": dta.F32}
HALF = {"bf16": 2.0 ** -8, "f32": U}

FORMS = [   # type, rows before a scored token, ids, width
    ("bf16", 8, 40, 64), ("bf16", 129, 33220, 192), ("bf16", 129, 47139, 64), ("bf16", 140, 40, 64), ("bf16", 16512, 131, 192),
    ("bf16", 100, 1290, 320), ("bf16", 16923, 42, 64), ("bf16", 33119, 42, 64), ("bf16", 33272, 43, 192),
    ("f32", 8, 40, 64), ("f32", 8, 33106, 64), ("f32", 809, 16881, 768), ("f32", 907, 16772, 192), ("f32", 1269, 195, 5440),
    ("f32", 1574, 2807, 832), ("f32", 8436, 1799, 192), ("f32", 17151, 129, 64), ("f32", 21772, 1817, 64),
    ("f32", 21778, 1382, 320), ("f32", 33871, 41, 64), ("f32", 41304, 928, 64),
    ("f32", 3491, 4611, 35264), ("f32", 754, 2529, 5632),
]


@pytest.mark.parametrize("dtype,rows,V,D", FORMS)
def test_every_kernel(dtype, rows, V, D):
    """A path whose last token has four children, two of them with the same id.  fp32 a second time with a number of 2^41 in
    one hidden row, under a column of zeros: multiplied on the fp32 instruction, wherever the first was not."""
    k = float(np.float32(0.8))
    p = dta.VocabParams(D, k, KIND[dtype])
    T = rows + 4
    rng = np.random.default_rng(rows + V)
    ids = rng.integers(0, V, size=T).astype(np.int32)
    ids[1], ids[-1] = V - 1, ids[-3]
    tok = dta.tokens_build(dta.tree_build([-1, 0, 0, 0, 0], [rows, 1, 1, 1, 1]), ids, V)
    assert tok.n_rows == rows and tok.n_scored == rows + 3
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(TORCH[dtype])
    h, w, d = mk(T, D), mk(V, D) * (2 / math.sqrt(D)), torch.randn(T, generator=g, device="cuda")
    start = torch.randn(V, D, generator=g, device="cuda")
    before = torch.arange(-1, T - 1, device="cuda")
    before[rows:] = rows - 1
    at, t = before[1:], torch.from_numpy(ids).cuda().long()[1:]
    for large in (False, True) if dtype == "f32" else (False,):
        if large:
            w[:, 0], h[:, 0] = 0.0, 0.0
            h[rows // 2, 0] = 2.0 ** 41
        hd, wd = h[:rows].double(), w.double()
        logp, lse = dta.tree_logprob_fwd(tok, p, h, w)
        z = k * (hd @ wd.t().contiguous())
        ref = torch.logsumexp(z, 1)
        zb = k * (hd.abs() @ wd.abs().t().contiguous()).amax(1) * (D * UM + U)
        lb = (128 + math.ceil(V / 128) / 64 + 12) * UM
        over = (lse[:rows].double() - ref).abs() - (zb + lb + 4 * U * ref.abs())
        assert over.max().item() <= 0, ("lse", large, over.max().item())
        want = z[at, t] - ref[at]
        over = (logp[1:].double() - want).abs() - (2 * zb[at] + lb + 8 * U * (want.abs() + ref[at].abs()))
        assert over.max().item() <= 0, ("logp", large, over.max().item())
        assert float(logp[0]) == 0 and (lse[rows:] == 0).all()
        # the gradient
        d_h, d_w = dta.tree_logprob_bwd(tok, p, h, w, lse, d)
        acc = start.clone()
        dta.tree_logprob_bwd(tok, p, h, w, lse, d, d_weight=acc, add=True, want_hidden=False)
        dd = d[1:].double()
        c = torch.zeros(rows, dtype=torch.float64, device="cuda").index_add_(0, at, dd)
        dz = torch.exp(z - ref[:, None]) * -c[:, None]
        size = dz.abs()
        dz.view(-1).index_add_(0, at * V + t, dd)
        size.view(-1).index_add_(0, at * V + t, dd.abs())
        del z
        r = 2 * U if dtype == "f32" else 2.0 ** -16 if rows <= 128 else 2.0 ** -8
        q = 2 * zb.max().item() + lb + 4 * U * ref.abs().max().item() + r
        want = k * (dz @ wd)
        b = (q + 2 * V * UM) * k * (size @ wd.abs())
        over = (d_h[:rows].double() - want).abs() - (b + HALF[dtype] * (want.abs() + b))
        assert over.max().item() <= 0, ("d_hidden", large, over.max().item())
        assert (d_h[rows:] == 0).all()
        want = k * (dz.t().contiguous() @ hd)
        b = (q + (2 * rows + 8) * UM) * k * (size.t().contiguous() @ hd.abs())
        over = (d_w.double() - want).abs() - (b + HALF[dtype] * (want.abs() + b))
        assert over.max().item() <= 0, ("d_weight", large, over.max().item())
        want += start
        over = (acc.double() - want).abs() - (b + 2 * U * (want.abs() + b))
        assert over.max().item() <= 0, ("d_weight added", large, over.max().item())
