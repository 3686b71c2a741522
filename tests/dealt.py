"""How dropout and the values of a held matrix deal rows to blocks and launches, written out again
(tests/test_dealt.py holds it against the library's own)."""


def dealt(groups):
    """(log2 of a row's threads in a block, a row's blocks) for a row of so many groups, one a thread."""
    log = min(8, max(0, (groups - 1).bit_length()))

    def chunks(l):
        return (groups + (1 << l) - 1) >> l

    for l in range(log - 1, 5, -1):
        if chunks(l) << l < chunks(log) << log:
            log = l
    return log, chunks(log)


def rows_a_launch(groups):
    log, chunks = dealt(groups)
    return max(1, (1 << 23) // chunks) << (8 - log)
