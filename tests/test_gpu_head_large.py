"""Heads (GPU) of vocabularies whose rows are worked on a block at a time: the same rows by themselves, and 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


# a block of 256 rows, of 512; as many tiles of all rows as would be 2^32 threads
@pytest.mark.parametrize("rows,vocab", [(600, (1 << 22) + 5), (1500, (1 << 21) + 1), (16384, (1 << 25) + 3)])
def test_blocks_of_rows(rows, vocab):
    import paper_2410_11415_amd as klay
    g = torch.Generator(device="cuda").manual_seed(rows)
    hidden = torch.randn((rows, 8), generator=g, device="cuda").bfloat16()
    weight = torch.randn((vocab, 8), generator=g, device="cuda").bfloat16()
    tokens = torch.randint(0, vocab, (rows, 2), generator=g, device="cuda")
    teacher = torch.randn((rows, 2), generator=g, device="cuda")
    r = klay.head_logprobs(hidden, weight, tokens, complement=True, entropy=True)
    loss = klay.head_distill(hidden, weight, tokens, teacher)
    for part in (slice(0, 300), slice(rows - 300, rows)):
        alone = klay.head_logprobs(hidden[part], weight, tokens[part], complement=True, entropy=True)
        for a, b in zip(r, alone):
            assert torch.equal(a[part], b)
        assert torch.equal(loss[part], klay.head_distill(hidden[part], weight, tokens[part], teacher[part]))
    some = torch.tensor([0, 255, 256, 511, 512, rows - 1], device="cuda")
    for i in some.tolist():
        x = (weight.double() * hidden[i].double()).sum(1)           # (the library's matrix-vector product is wrong at 2^25 rows of 64 bits)
        lp = torch.log_softmax(x, 0)
        p = lp.exp()
        # (sums of up to 2^25 terms in fp32: a tile's of 65536, then thousands of tiles', each off by 2^-24 a step; entropies of up to 17)
        off = 2.0 ** -24 * (256 + vocab / 65536)
        assert float((r.logp[i].double() - lp[tokens[i]]).abs().max()) <= off + 2.0 ** -22 * 30
        assert float((r.neg[i].double() - torch.log1p(-p[tokens[i]])).abs().max()) <= 2.0 ** -22
        assert abs(float(r.entropy[i]) - float(-(p * lp).sum())) <= 30 * off
