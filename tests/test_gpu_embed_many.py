"""The embedding's gradient of many tokens: more groups of 64 ids for a wave than a mask of 64 bits has bits, at the
numbers of groups where a bit comes to stand for twice as many."""
import pytest
import torch

from sequence_util import TYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    return pkg


# A block of the sort has eight waves; tables of more than 262144 rows and up to 4096 tokens are sorted in one share, small
# tables in eight: 64, 65, 128, 129, 257 groups of 64 tokens a wave, and whole numbers of tokens around them.
GROUPS = [64, 65, 128, 129, 257]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab,shares", [(300000, 1), (1000, 8), (70000, 4)])
@pytest.mark.parametrize("groups", GROUPS)
@pytest.mark.parametrize("less", [0, 63, 511])
def test_gradient(lb, groups, vocab, shares, less, dtype):
    n, dim = groups * 64 * 8 * shares - less, 4
    g = torch.Generator().manual_seed(n)
    kind = torch.int32 if groups % 2 else torch.int64
    ids = torch.randint(0, vocab, (n,), generator=g)
    ids[torch.rand(n, generator=g) < 0.3] = vocab // 2          # a row in every group
    ids[-1] = vocab - 1                                         # one in the last group alone
    dout = torch.randn(n, dim, generator=g).to(TYPES[dtype])
    want = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, ids, dout.double())
    size = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, ids, dout.double().abs())
    count = torch.bincount(ids, minlength=vocab)[:, None]
    got = lb.lbscan_embed_bwd(ids.to(kind).cuda(), dout=dout.cuda(), vocab=vocab).double().cpu()
    # a row's tokens are added in pieces of 32, the pieces in eight shares: 32 + pieces / 8 + 8 roundings of at most the sum of
    # their sizes, then one to the storage type
    bound = (32 + count / 256 + 8) * 2.0 ** -24 * size + (want.abs() * 2.0 ** -8 if dtype == "bf16" else 0)
    assert bool(((got - want).abs() <= bound).all()), f"{n} tokens of {vocab}"
