"""Token embedding of more tokens than one launch has threads for (32 bits of them along an axis of its grid)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

MANY = (1 << 28) + 1000


@pytest.fixture(scope="module")
def lb():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2506_15976_amd as pkg
    pkg.load()
    yield pkg
    torch.cuda.empty_cache()          # (the blocks are large)


@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
def test_lookup(lb, kind):
    weight = torch.randn(300, 2, device="cuda").bfloat16()
    ids = torch.randint(0, 300, (MANY,), device="cuda", dtype=kind)
    out = torch.full((MANY, 2), 7.0, device="cuda", dtype=torch.bfloat16)
    lb.lbscan_embed_fwd(ids, weight, out=out)
    for part in torch.arange(0, MANY, 1 << 24).tolist():
        some = slice(part, part + (1 << 24))
        assert torch.equal(out[some], weight[ids[some].long()]), part


def test_gradient(lb):
    """Ones: their sums are the numbers of tokens, exact in 32 bits."""
    vocab = 70000
    ids = torch.randint(0, vocab, (MANY,), device="cuda", dtype=torch.int32)
    got = lb.lbscan_embed_bwd(ids, dout=torch.ones(MANY, 1, device="cuda"), vocab=vocab)
    want = torch.zeros(vocab, dtype=torch.int64, device="cuda")
    for part in ids.split(1 << 24):
        want += torch.bincount(part, minlength=vocab)
    assert torch.equal(got[:, 0].long(), want)
