"""Words of memory that the grouped products load of operands off 16-byte boundaries (host code on its own; no GPU)."""
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def words(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("words") / "harness")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(HERE, "grouped_words_harness.cpp"), "-o", exe], check=True)

    def run(cases, what="w"):
        out = subprocess.run([exe], input="".join(f"{what} {a} {v}\n" for a, v in cases), capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(cases)
        return [[int(w) for w in line.split()] for line in out]
    return run


def test_every_word_holds_a_valid_half_and_every_valid_half_has_its_word(words):
    cases = [(4096 + 2 * shift, valid) for shift in range(16) for valid in range(-200, 12)]
    for (address, valid), got in zip(cases, words(cases)):
        halves = [address + 2 * e for e in range(max(0, min(valid, 8)))]
        assert got == sorted({h & ~3 for h in halves}), (address, valid)


@pytest.mark.parametrize("rows, width, ld, base", [(1, 767, 767, 0), (129, 767, 767, 2), (65, 5, 5, 0), (3, 9, 1001, 6)])
def test_a_tile_of_rows_stays_inside_of_its_matrix(words, rows, width, ld, base):
    """Every unit of 128-row tiles over a matrix whose allocation ends with its last element: rows behind the last and columns behind the width included."""
    start, end = 1 << 20, (1 << 20) + base + 2 * ((rows - 1) * ld + width)
    cases = []
    for row in range((rows + 127) // 128 * 128):
        for col in range(0, (width + 63) // 64 * 64, 8):
            cases.append((start + base + 2 * (row * ld + col), width - col if row < rows else 0))
    for (address, valid), got in zip(cases, words(cases)):
        for w in got:
            # a word is inside where one of its halves is: allocations begin and end on words
            assert start + base - 2 <= w < end, (address, valid)


def test_parts_of_images_longer_than_31_bits(words):
    """Images of 1024 weights of 1024 x 1024 fp32 elements and more: part 1 lies 2^31 bytes behind part 0, part 2 twice as far."""
    cases = [(k, apart) for apart in (16384, (1 << 30) + 16, (1 << 31) - 16, 1 << 31, 3 << 31, 1 << 38) for k in range(3)]
    assert words(cases, "p") == [[k * apart] for k, apart in cases]


def test_each_copy_in_flight_is_known_by_its_barrier_and_phase(words):
    """Sequences of copies, those with rows behind an item at random places: the k-th use of a barrier ends its phase k, of parity k mod 2."""
    rng = random.Random(3)
    cases = [(slots, 1 << n | rng.getrandbits(n) if n else 1) for slots in (1, 2, 4, 6, 8) for n in (0, 1, 2, 5, 7, 12, 30, 55) for _ in range(20)]
    for (slots, flags), got in zip(cases, words(cases, "c")):
        tails = [flags >> i & 1 for i in range(flags.bit_length() - 1)]
        want = []
        for i in range(max(0, len(tails) - slots), len(tails)):
            before = range(i % slots, i, slots)            # earlier copies of this slot
            uses = sum(tails[j] for j in before) if tails[i] else len(before)
            want += [i % slots, tails[i], uses % 2]
        assert got == want, (slots, flags)
