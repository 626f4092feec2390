"""The whole numbers of csrc/chunk_rows.h that say how blocks are given out: those of the model in
test_chunk_shares_cpu.py are the kernel's, line by line where it copies one, and the largest
sizes that duo_attention_chunk takes are within them."""

import os
import re

import pytest

import test_chunk_shares_cpu as M
from paper_2506_20194_amd import build as B

TEXT = re.sub(r"\s+", " ", re.sub(r"//.*", "", open(os.path.join(B.CSRC, "chunk_rows.h")).read()))
MOST = 1 << 30  # tokens, and new tokens times heads


def number(name):
    return eval(re.search(r"\b" + name + r" = ([^,;]+)[,;]", TEXT).group(1).replace("INT32_MAX", str(2 ** 31 - 1)))


def test_the_model_has_the_kernels_numbers():
    assert (M.QB, M.COST, M.LEAST, M.SNAP) == tuple(number("kRows" + n) for n in ("QB", "Cost", "Min", "Snap"))
    assert M.KB == number("KB")


@pytest.mark.parametrize("line", [
    "dealt = a.deal ? nb / a.deal * a.deal : 0; nb -= dealt; first = max(len - lq, 0);",
    "(int)min((int64_t)a.window + a.sinks + a.qpb + 192, ",
    "linear = most < first ? 0 : min((most - first) / a.qpb, nb);",
    "return (n < linear ? first + (n + 1) * a.qpb : most) + kRowsCost;",
    "return m * (first + kRowsCost) + m * (m + 1) / 2 * a.qpb + (int64_t)(n - m) * ((int64_t)most + kRowsCost);",
    "(int)min((int64_t)gridDim.x, (total + kRowsMin - 1) / kRowsMin);",
    "auto begin = [&](int i) { return i * size + min(i, more); };",
    "const int64_t cut = more * (size + 1); return u < cut ? (int)rows_div(u, size + 1) : more + (int)rows_div(u - cut, size);",
    "(int)min((int64_t)min(kRowsSnap, c / 2), size / 2);",
    "p.at <= near(c) ? u - p.at : c - p.at <= near(c) ? u - p.at + c : u",
    "q.nb + q.dealt - 1 - (round * a.deal + (round & 1 ? a.deal - 1 - j : j))",
    "const int sinks = same((min(a.sinks, first) + KB - 1) / KB), from = same(max(first / KB, sinks));",
    "pos_end < 0 ? 0 : sinks + (pos_end + KB) / KB - from",
    "min(max((x - kRowsCost + KB - 1) / KB, 0), tiles)",
    "block + min(kRowsCost + (tiles - 1) * KB + 1, cost - near(cost)); ",
    "share_of(end - 1) - share + 1",
])
def test_the_model_has_the_kernels_lines(line):
    """A line that changes here has to change in the model too."""
    assert line in TEXT


def test_largest_sizes():
    """A block that is dealt out has all of its tiles, and without a window every query sees every token before it."""
    most = number("kRowsAll")
    tiles = MOST // M.KB + 3  # of the sinks and of the window, both rounded
    assert (most - M.COST + M.KB - 1) // M.KB >= tiles and most + M.KB - 1 - M.COST < 2 ** 31
    back = number("kRowsBack")
    assert MOST - 1 - back < 0 and -MOST - back >= -2 ** 31  # key 0 from the last position; no overflow at the first
