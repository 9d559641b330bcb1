"""GPU tests of the vocabulary ends at the limits of their sizes and lifetimes: calls of more logits than one launch has
threads for, and token tables given back behind calls that have not run.  Bounds as in tests/test_gpu_vocab.py."""
import math

import numpy as np
import pytest
import torch

import paper_2602_00482_amd as dta

pytestmark = pytest.mark.gpu

U, UM = 2.0 ** -24, 2.0 ** -23
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
KIND = {"bf16": dta.BF16, "f32": dta.F32}


@pytest.mark.parametrize("dtype,rows,V", [("bf16", 2 ** 21, 2 ** 18 + 300), ("f32", 2 ** 20 + 3, 2 ** 18 + 300)])
def test_more_logits_than_a_launch_has_threads_for(dtype, rows, V):
    """2^39 logits (f32: 2^38) in launches over parts of the vocabulary: 600 rows, the first and the last among them,
    against 64 bits."""
    D = 64
    rng = np.random.default_rng(rows)
    ids = rng.integers(0, V, size=rows + 1).astype(np.int32)
    ids[1], ids[-1] = 0, V - 1
    tok = dta.tokens_build(dta.tree_build([-1], [rows + 1]), ids, V)
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(TORCH[dtype])
    h, w = mk(rows + 1, D), mk(V, D) * (2 / math.sqrt(D))
    logp, lse = dta.tree_logprob_fwd(tok, dta.VocabParams(D, 1.0, KIND[dtype]), h, w)
    at = np.unique(np.concatenate(([0, rows - 1], rng.integers(0, rows, size=600))))
    t = torch.from_numpy(at).cuda()
    hd, wd = h[t].double(), w.double()
    z = hd @ wd.t().contiguous()
    ref = torch.logsumexp(z, 1)
    want = z[torch.arange(len(at), device="cuda"), torch.from_numpy(ids[at + 1]).cuda().long()] - ref
    zb = float((hd.abs() @ wd.abs().t().contiguous()).max()) * (D * UM + U)
    lb = (128 + math.ceil(V / 128) / 64 + 12) * UM
    assert ((lse[t].double() - ref).abs() <= zb + lb + 4 * U * ref.abs()).all()
    assert ((logp[t + 1].double() - want).abs() <= 2 * zb + lb + 8 * U * (want.abs() + ref.abs())).all()
    assert float(logp[0]) == 0 and float(lse[-1]) == 0
    assert bool(torch.isfinite(lse).all()) and float(lse[:-1].min()) > math.log(V) - 1   # (every row was written)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tables_given_back_behind_calls_that_have_not_run(dtype):
    """Calls on two streams behind long products; their tables are destroyed while both streams are still at the products, and
    the memory of that size is then asked for until there is no more of it.  Uploads may share a hardware queue with one of the
    streams and so wait for it: pairs of streams are tried until one pair is seen still at work behind the uploads."""
    rows, V, D = 6000, 9000, 256
    rng = np.random.default_rng(3)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda").to(TORCH[dtype])
    h, w, d_x, d = mk(rows, D), mk(V, D) * 0.1, mk(rows, D), torch.randn(rows, generator=g, device="cuda")
    big = torch.randn(8192, 8192, device="cuda").bfloat16()
    out = [torch.empty_like(big) for _ in range(2)]
    p = dta.VocabParams(D, 1.0, KIND[dtype])
    tree = dta.tree_build([-1, 0, 0], [rows // 2, rows // 4, rows // 4])
    ids = rng.integers(0, V, size=rows).astype(np.int32)
    build = lambda x: dta.tokens_build(tree, x, V)

    def calls(tok):
        x = dta.tree_embed_fwd(tok, p, w)
        logp, lse = dta.tree_logprob_fwd(tok, p, h, w)
        return (x, logp, lse, *dta.tree_logprob_bwd(tok, p, h, w, lse, d), dta.tree_embed_bwd(tok, p, d_x))

    first = build(ids)
    ref = calls(first)
    torch.mm(big, big, out=out[0])
    torch.cuda.synchronize()
    overlapped = False
    for attempt in range(6):
        tok, streams = build(ids), [torch.cuda.Stream(), torch.cuda.Stream()]
        tok.prepare()
        others = [build(np.roll(ids, 1 + k)) for k in range(8)]
        got, ends = [], []
        for s, o in zip(streams, out):
            with torch.cuda.stream(s):
                for _ in range(40):                       # some 30 ms
                    torch.mm(big, big, out=o)
                got.append(calls(tok))
                ends.append(torch.cuda.Event())
                ends[-1].record(s)
        tok.destroy()
        assert not any(e.query() for e in ends), "the products were over before the tables were given back"
        for o in others:
            o.prepare()
        overlapped = not any(e.query() for e in ends)
        torch.cuda.synchronize()
        for one in got:
            for a, b in zip(ref, one):
                assert torch.equal(a, b)
        if overlapped:
            break
    assert overlapped


@pytest.mark.parametrize("dtype,T,V,D", [("bf16", 67001, 97000, 2112), ("f32", 33001, 48000, 2112), ("bf16", 33001, 49001, 4160)])
def test_embeddings_larger_than_the_memory_side_cache(dtype, T, V, D):
    """x of 256 MiB and more and a table's gradient of 384 MiB and more, with long sums, are stored past the cache."""
    size = torch.tensor([], dtype=TORCH[dtype]).element_size()
    assert T * D * size >= 256 << 20 and V * D * size >= 384 << 20
    rng = np.random.default_rng(5)
    ids = rng.integers(0, V, size=T).astype(np.int32)
    ids[rng.random(T) < 0.02] = V - 1
    tok = dta.tokens_build(dta.tree_build([-1], [T]), ids, V)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    table, d_x = (torch.randn(n, D, generator=g, device="cuda").to(TORCH[dtype]) for n in (V, T))
    p, at = dta.VocabParams(D, 1.25, KIND[dtype]), torch.from_numpy(ids).cuda().long()
    x = dta.tree_embed_fwd(tok, p, table)
    assert torch.equal(x, (table[at].float() * 1.25).to(TORCH[dtype]))   # (one product in fp32, one rounding)
    d_table = dta.tree_embed_bwd(tok, p, d_x)
    n = torch.bincount(at, minlength=V).double()[:, None]
    ref = torch.zeros(V, D, device="cuda", dtype=torch.float64).index_add_(0, at, 1.25 * d_x.double())
    sums = torch.zeros(V, D, device="cuda", dtype=torch.float64).index_add_(0, at, 1.25 * d_x.double().abs())
    b = (n + 1) * U * sums
    half = 2.0 ** -8 if dtype == "bf16" else U
    over = (d_table.double() - ref).abs() - (b + half * (ref.abs() + b))
    assert over.max().item() <= 0, over.max().item()
    assert (d_table[n[:, 0] == 0] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V,D", [(39, 300, 64), (300, 33000, 64), (1100, 16500, 64), (18700, 290, 320)])
def test_infinite_logits_and_nan_stay_in_their_rows(dtype, rows, V, D):
    """In each form of the logits: a row of -inf has lse -inf, one logit of +inf gives lse +inf and logp -inf elsewhere, NaN
    gives NaN; every other row is as without them."""
    rng = np.random.default_rng(rows)
    ids = rng.integers(0, V, size=rows + 1).astype(np.int32)
    ids[10] = 5
    tok = dta.tokens_build(dta.tree_build([-1], [rows + 1]), ids, V)
    p = dta.VocabParams(D, 1.0, KIND[dtype])
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    h = torch.randn(rows + 1, D, generator=g, device="cuda").to(TORCH[dtype])
    w = (torch.randn(V, D, generator=g, device="cuda") * (2 / math.sqrt(D))).to(TORCH[dtype])
    h[:, 0], w[:, 0] = 0.0, 1.0
    logp, lse = dta.tree_logprob_fwd(tok, p, h, w)
    w[77, 0] = 1.0e38
    h[5, 0], h[6, 0], h[9, 0], h[rows - 1, 0] = -math.inf, math.nan, 1.0e38, math.nan
    logp2, lse2 = dta.tree_logprob_fwd(tok, p, h, w)
    assert float(lse2[5]) == -math.inf and math.isnan(float(lse2[6])) and float(lse2[9]) == math.inf
    assert math.isnan(float(lse2[rows - 1])) and math.isnan(float(logp2[rows])) and float(logp2[10]) == -math.inf
    rest = torch.ones(rows + 1, dtype=torch.bool, device="cuda")
    rest[[5, 6, 9, rows - 1]] = False
    # (fp32 with NaN is multiplied on the fp32 instruction: other roundings)
    hd, wd = h[rest][:, 1:].double(), w[:, 1:].double()
    zb = float((hd.abs() @ wd.abs().t().contiguous()).max()) * (D * UM + U)
    lb = (128 + math.ceil(V / 128) / 64 + 12) * UM
    bound = 0 if dtype == "bf16" else 2 * (zb + lb)
    assert ((lse2 - lse).abs()[rest] <= bound).all()
    after = torch.ones(rows + 1, dtype=torch.bool, device="cuda")
    after[[6, 7, 10, rows]] = False
    assert ((logp2 - logp).abs()[after] <= 2 * bound).all()
