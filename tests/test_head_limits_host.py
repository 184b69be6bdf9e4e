"""Host-only checks of the vocabulary head's plan at the largest sizes that it takes."""
from paper_2502_19864_amd import binding as B

MIB = 1 << 20


def plan(rows, d, vocab, dtype=B.BF16):
    return B.ringada_vocab_plan(B.VocabDesc(dtype, rows, d, vocab))


def test_the_largest_plans_are_by_the_same_rule():
    """The tile of the logits is chosen by its cost where rows times classes are most, too: a block of classes more or
    less leaves the partial sums' width, so the workspace grows by that block's."""
    for d in (8, 64, 4096):
        most, less = plan(1 << 23, d, 1 << 22), plan(1 << 23, d, (1 << 22) - 128)
        for a, b in zip(most, less):
            assert 0 <= a - b < 8 * MIB, (d, a - b)


def test_plans_of_few_rows():
    """Without gradients, up to 32 rows in bf16 whose h fits the LDS: 4 KiB a row for the loss, 6 for the next token, and
    a block for each array."""
    for n, d, vocab in ((1, 8, 40), (5, 4096, 32000), (15, 4096, 32000), (7, 8192, 32000), (3, 16384, 300), (32, 64, 1 << 22)):
        forward, _, following = plan(n, d, vocab)
        assert 0 < forward <= 4096 * n + 512 and 0 < following <= 6144 * n + 512, (n, d, vocab, forward, following)
    for n, d in ((33, 64), (16, 4096), (8, 8192), (4, 16384)):
        assert plan(n, d, 32000)[0] >= 2 * n * d  # a copy of h
