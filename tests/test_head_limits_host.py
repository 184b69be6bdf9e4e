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
