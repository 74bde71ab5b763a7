"""Calls of the loss in bf16 that take each of the ways in which what rounding the targets' slopes leaves is added to the gradients:
dweight from sums that are cut into parts ("cut") or from whole ones, of the pieces before the last and of the last one; dx from a table
whose rows are read in place, read loose, or copied."""

# tokens, rows of the table, columns, part of the tokens that is ignored; dweight of the pieces before the last, of the last; the table's rows
CALLS = [
    (4000, 3000, 256, 0.0, None, "cut", "in place"),
    (1024, 65600, 256, 0.1, None, "whole", "in place"),             # tiles fill the machine
    (300, 3000, 256, 0.2, None, "whole", "in place"),               # too few steps for a second part
    (511, 1000, 128, 0.1, None, "whole", "in place"),               # planned for two parts, of which the live tokens need one
    (300, 1000, 70, 0.0, None, "whole", "copied"),
    (3000, 900, 130, 0.1, None, "cut", "copied"),
    (64, 500, 64, 0.0, None, "whole", "in place"),
    (40, 2000, 128, 0.2, None, "whole", "in place"),
    (64, 500, 65, 0.0, None, "whole", "loose"),
    (50, 700, 130, 0.2, None, "whole", "loose"),
    (16384, 40000, 512, 0.0, "whole", "cut", "in place"),
]


def live(tokens, ignored):
    """The tokens that are not ignored: the first ones of every ten are."""
    return [t for t in range(tokens) if t % 10 >= round(10 * ignored)]
