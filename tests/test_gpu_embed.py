"""Token embedding on the GPU: lookups bit for bit, the gradient against the 64-bit reference for tokens that are
absent, rare, common and alone in the batch."""
import numpy as np
import pytest
import torch

import sequence_reference as ref
from sequence_util import TYPES, off_by_one, to_numpy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


def ids_of(kind, n, vocab, seed=0):
    g = torch.Generator().manual_seed(seed + n)
    if kind == "zipf":
        ids = (torch.exp(torch.rand(n, generator=g, dtype=torch.float64) * np.log(vocab + 1)) - 1).long().clamp(0, vocab - 1)
    elif kind == "uniform":
        ids = torch.randint(0, vocab, (n,), generator=g)
    elif kind == "one":
        ids = torch.full((n,), vocab - 1)
    else:                                            # padding and numbers that are no rows among others
        ids = torch.randint(-2, vocab + 2, (n,), generator=g)
        ids[::5] = torch.iinfo(torch.int32).max
        ids[::7] = torch.iinfo(torch.int32).min
    return ids


def check_gradient(lb, ids, vocab, dim, dtype, scale=1.5, seed=0):
    g = torch.Generator().manual_seed(seed)
    dout = torch.randn(ids.numel(), dim, generator=g).to(TYPES[dtype]).cuda().view(*ids.shape, dim)
    got = lb.lbscan_embed_bwd(ids, dout=dout, vocab=vocab, scale=scale)
    want = ref.embed_bwd(ids.cpu().numpy(), to_numpy(dout), vocab, scale)
    # sums of k terms in 32 bits: (k + 2) roundings of at most the sum of their sizes, then one to the storage type
    size = ref.embed_bwd(ids.cpu().numpy(), np.abs(to_numpy(dout)), vocab, scale)
    count = np.bincount(ids.cpu().numpy().reshape(-1).clip(-1, vocab) + 1, minlength=vocab + 2)[1:vocab + 1, None]
    bound = (np.minimum(count, 100) + 2) * 2.0 ** -24 * size + (np.abs(want) * 2.0 ** -8 if dtype == "bf16" else 0)
    assert got.shape == (vocab, dim) and got.dtype == TYPES[dtype]
    off = np.abs(to_numpy(got) - want) - bound
    assert off.max() <= 0, f"off by {off.max():.2e} more than the bound"


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 5, 3), (3, 7, 8), (5, 100, 7), (64, 300, 64), (130, 513, 100),
                                         (1000, 40, 385), (17, 1000, 2049)])
def test_lookup(lb, n, vocab, dim, wide, dtype):
    g = torch.Generator().manual_seed(n)
    weight = torch.randn(vocab, dim, generator=g).to(TYPES[dtype]).cuda()
    for kind in ("uniform", "outside"):
        ids = ids_of(kind, n, vocab).to(torch.int64 if wide else torch.int32).cuda()
        scale = 0.37
        out = lb.lbscan_embed_fwd(ids, weight, scale=scale)
        ok = (ids >= 0) & (ids < vocab)
        want = torch.where(ok[:, None], weight[torch.where(ok, ids, 0).long()].float() * np.float32(scale), 0.0).to(TYPES[dtype])
        assert torch.equal(out, want), kind


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["zipf", "uniform", "one", "outside"])
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 300, 5), (31, 7, 8), (32, 1, 64), (33, 2, 65), (64, 600, 3),
                                         (500, 257, 100), (2000, 3, 24), (3000, 5000, 33), (1025, 131, 1030),
                                         (5000, 140000, 9)])
def test_gradient(lb, n, vocab, dim, kind, dtype):
    check_gradient(lb, ids_of(kind, n, vocab).cuda(), vocab, dim, dtype)


@pytest.mark.parametrize("n", [1, 63, 64, 65, 1023, 1024, 1025, 4096, 4097, 20011])
def test_gradient_token_counts(lb, n):
    check_gradient(lb, ids_of("zipf", n, 700).to(torch.int32).cuda(), 700, 16, "fp32")


def test_a_row_of_the_table_beyond_32_bits(lb):
    """Element offsets of the table pass 2^31: 2.2 billion elements, 4.3 GB."""
    vocab, dim = 70000, 31000
    weight = torch.zeros(vocab, dim, dtype=torch.bfloat16, device="cuda")
    last = torch.randn(dim, device="cuda").bfloat16()
    weight[-1] = last
    ids = torch.tensor([vocab - 1, 0], device="cuda")
    out = lb.lbscan_embed_fwd(ids, weight)
    assert torch.equal(out[0], last) and not out[1].any()
    del weight
    dout = torch.randn(2, dim, device="cuda").bfloat16()
    g = lb.lbscan_embed_bwd(ids, dout=dout, vocab=vocab)
    assert torch.equal(g[-1], dout[0]) and torch.equal(g[0], dout[1]) and not g[1:-1:997].any()


def test_nan_stays_with_its_token(lb):
    weight = torch.randn(10, 20, device="cuda")
    weight[0] = float("nan")
    out = lb.lbscan_embed_fwd(torch.tensor([-1, 0, 3, 10], device="cuda"), weight)
    assert not out[0].any() and torch.isnan(out[1]).all() and torch.equal(out[2], weight[3]) and not out[3].any()
    dout = torch.randn(4, 20, device="cuda")
    dout[0], dout[3] = float("nan"), float("inf")     # of padding
    g = lb.lbscan_embed_bwd(torch.tensor([-1, 0, 3, 10], device="cuda"), dout=dout, vocab=10)
    assert torch.isfinite(g).all() and torch.equal(g[3], dout[2])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim", [5, 12, 100])
def test_alignment(lb, dim, dtype):
    ids = ids_of("zipf", 200, 50).cuda()
    weight = torch.randn(50, dim, device="cuda").to(TYPES[dtype])
    dout = torch.randn(200, dim, device="cuda").to(TYPES[dtype])
    a = lb.lbscan_embed_fwd(off_by_one(ids), off_by_one(weight), out=off_by_one(torch.zeros(200, dim, device="cuda", dtype=TYPES[dtype])))
    assert torch.equal(a, lb.lbscan_embed_fwd(ids, weight))
    assert torch.equal(lb.lbscan_embed_bwd(ids, dout=off_by_one(dout), vocab=50), lb.lbscan_embed_bwd(ids, dout=dout, vocab=50))


def test_empty_and_shapes(lb):
    weight = torch.randn(9, 4, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert lb.lbscan_embed_fwd(none, weight).shape == (0, 4)
    assert not lb.lbscan_embed_bwd(none, dout=torch.empty(0, 4, device="cuda"), vocab=9).any()
    ids = torch.randint(0, 9, (3, 5), device="cuda")
    assert torch.equal(lb.lbscan_embed_fwd(ids, weight), weight[ids])
    assert lb.lbscan_embed_fwd(torch.tensor(3, device="cuda"), weight).shape == (4,)
    check_gradient(lb, ids, 9, 4, "fp32")


def test_autograd_bits_and_streams(lb):
    from paper_2506_15976_amd.autograd import token_embedding
    ids = ids_of("zipf", 6000, 900).view(6, 1000).cuda()
    weight = torch.randn(900, 72, device="cuda", requires_grad=True)
    out = token_embedding(ids, weight, scale=3.0)
    dout = torch.randn_like(out)
    g, = torch.autograd.grad(out, weight, dout)
    again = lb.lbscan_embed_bwd(ids, dout=dout, vocab=900, scale=3.0)
    assert torch.equal(g, again)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    other = lb.lbscan_embed_bwd(ids, dout=dout, vocab=900, scale=3.0, stream=s)
    s.synchronize()
    assert torch.equal(other, g)


def test_gradient_against_differences(lb):
    ids = ids_of("zipf", 100, 30).cuda()
    weight, dout = torch.randn(30, 12, device="cuda"), torch.randn(100, 12, device="cuda")
    g = lb.lbscan_embed_bwd(ids, dout=dout, vocab=30, scale=2.0)
    d = torch.randn(30, 12, device="cuda")
    loss = lambda w: float((lb.lbscan_embed_fwd(ids, w, scale=2.0).double() * dout).sum())  # noqa: E731
    want = (loss(weight + d) - loss(weight - d)) / 2         # (linear: any step)
    assert abs(float((g.double() * d).sum()) - want) <= 1e-4 * (abs(want) + 10)
