"""How the passes over fp32 arrays for pairs of fp16 values go through them (as gpga_pack.cuh computes it): every chunk of eight columns
of every row is taken once, and what is noted for columns and rows stays inside its array."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2105_09080_b200" / "csrc"


def slice_rows(rows, chunks, batches, sms=148):
    piece = 8
    while piece < 1024:
        units = batches * -(-rows // piece) * -(-chunks // 32)
        if not (piece < 64 and units > sms * 5 // 2 or units > sms * 16):
            break
        piece *= 2
    return piece


def places(unit, rows, chunks, piece):
    """(batch, row, chunk, column of shared memory) that the 256 threads of a block take of a unit."""
    strips, slices = -(-chunks // 32), -(-rows // piece)
    t, strip = unit // strips, unit % strips
    batch, first = t // slices, t % slices * piece
    lanes = 32 if chunks > 16 else 16 if chunks > 8 else 8 if chunks > 4 else 4 if chunks > 2 else chunks
    end = min(first + piece, rows)
    for thread in range(256):
        chunk = strip * 32 + (thread & (lanes - 1))
        for row in range(first + thread // lanes, end, 256 // lanes):
            if chunk < chunks:
                yield batch, row, chunk, (thread & (lanes - 1)) * 8


@pytest.mark.parametrize("rows,chunks,batches", [(1, 1, 1), (64, 1, 3), (300, 2, 2), (65, 3, 2), (130, 4, 1), (70, 5, 2), (200, 9, 1), (129, 16, 1), (100, 17, 2),
                                                 (77, 32, 2), (1000, 33, 1), (63, 100, 3)])
def test_every_chunk_is_taken_once(rows, chunks, batches):
    piece = slice_rows(rows, chunks, batches)
    units = batches * -(-rows // piece) * -(-chunks // 32)
    seen = set()
    for unit in range(units):
        for batch, row, chunk, column in places(unit, rows, chunks, piece):
            assert batch < batches and row < rows and 0 <= column <= 248 and chunk * 8 == unit % -(-chunks // 32) * 256 + column
            assert (batch, row, chunk) not in seen
            seen.add((batch, row, chunk))
    assert len(seen) == batches * rows * chunks


def test_exponents_are_those_of_normal_numbers():
    """A power's exponent is held, negated, in a byte; halves of two of them, added, are exponents of normal fp32 numbers, and the largest
    value of a row comes to 2^14 .. 2^15 wherever fp32 has such a power."""
    source = (CSRC / "gpga_pack.cuh").read_text()
    low, bias, most = map(int, re.search(r"min\((\d+) \+ (\d+) - \(int\)\(peak >> 23\), (\d+)\)", source).groups())
    kept = [-min(low + bias - field, most) for field in range(255)]       # of the exponent field of the largest finite value
    assert all(-128 <= e <= 127 for e in kept)
    for field, e in enumerate(kept):
        if field >= low + bias - most:
            assert field - bias - e == low
    halves = [h for e in kept for h in (e >> 1, e - (e >> 1))]
    assert min(halves) * 2 >= -126 and max(halves) * 2 <= 127


def row_units(rows, chunks):
    """(row, chunk) that the 256 threads of a block hold of each unit of short rows: four chunks each."""
    threads = 1
    while threads < 256 and threads < chunks:
        threads *= 2
    slots = 4 if chunks > 512 else 2 if chunks > 256 else 1
    per = 4 // slots * (256 // threads)
    for unit in range(-(-rows // per)):
        for thread in range(256):
            for q in range(4):
                row, chunk = unit * per + thread // threads + q // slots * (256 // threads), (thread & (threads - 1)) + threads * (q & (slots - 1))
                if row < rows and chunk < chunks:
                    yield row, chunk
        if chunks > 1024:       # the rest of the one row
            for thread in range(256):
                for chunk in range(thread + 1024, chunks, 256):
                    yield unit, chunk


@pytest.mark.parametrize("rows,chunks", [(1, 1), (1025, 1), (700, 2), (300, 3), (130, 17), (65, 33), (33, 64), (9, 200), (5, 256), (5, 257), (3, 512), (3, 513), (2, 1024),
                                         (2, 1025), (3, 1700)])
def test_every_chunk_of_short_rows_is_taken_once(rows, chunks):
    seen = list(row_units(rows, chunks))
    assert len(seen) == rows * chunks and len(set(seen)) == rows * chunks
