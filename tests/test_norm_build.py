"""Which kernels of the norms around a block are built: those that some call reaches, and none that spills."""
import os
import re


def test_the_build_refuses_norms_that_spill():
    from paper_2307_11339_amd import _build as B
    kernel, piece = B.NO_SPILL["block_norm.hip"]
    source = open(os.path.join(B.CSRC, "block_norm.hip")).read()
    assert re.search(r"__global__[^;{]*\b%s\(" % kernel, source, re.S) and piece == ""


def _pieces_a_thread(width, groups, vec, rows):
    """norm_slots and norm_divide of block_norm.hip, for 256 compute units."""
    up = lambda n: 1 << (n - 1).bit_length()
    pieces = width // groups // vec
    third = -(-pieces // 3)
    deep = 3 if groups > 1 and pieces <= 64 and 5 * up(pieces) >= 18 * up(third) else 1
    in_group = third if deep == 3 else pieces
    lanes = up(in_group) if in_group <= 32 or (groups > 1 and in_group <= 64) else -(-in_group // 64) * 64
    slots = lanes * groups
    if slots <= 32 and slots & (slots - 1) == 0 and deep == 1:
        return 1, 1
    chunks = -(-slots // 64)
    waves = -(-chunks // (1 if deep == 3 else 2))
    while waves < chunks and waves < 8 and rows * waves < 1024:
        waves += 1
    waves = min(waves, 8)
    return waves, -(-chunks // waves) * deep


def test_pieces_a_thread_of_every_width():
    """bf16 rows, and rows that are one group, never have more than eight: no kernel is built for more.  Where one wave has the
    row there are at most two, or three of one group."""
    for vec in (4, 8):
        most = {True: 0, False: 0}
        for width in range(vec, 16385, vec):
            for groups in [g for g in range(1, 513) if width % g == 0]:
                if width // groups % vec or (groups > 1 and width // groups < 32):
                    continue
                for rows in (1, 60, 5000):
                    waves, n = _pieces_a_thread(width, groups, vec, rows)
                    assert waves > 1 or n <= 3
                    most[groups > 1] = max(most[groups > 1], n)
        assert most[False] <= 8 and most[True] <= (8 if vec == 8 else 16)
