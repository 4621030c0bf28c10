"""Key tiles of a tile of query rows as attention over pages forms them (csrc/paged_attn.h, compiled for the host), against whole
numbers without a width: ragged lengths, rows before the first token, windows up to the largest number the call takes."""
import subprocess

import pytest

from paper_2602_23592_amd import build

PROGRAM = r"""
#include <cstdio>
#include "paged_attn.h"
using namespace keep;

template <int TR, int KT>
void spans(const PagedArgs& a, const PagedSeq& q) {
  for (int t = 0; t < paged_tiles<TR>(a, q); ++t) {
    int first, units;
    paged_span<TR, KT>(a, q, t, first, units);
    printf(" %d %d", first, units);
  }
  printf("\n");
}

int main() {
  int tr, rep, window, rows, len;
  while (scanf("%d %d %d %d %d", &tr, &rep, &window, &rows, &len) == 5) {
    PagedArgs a{};
    a.rep = rep;
    a.window = window;
    a.by_rep = fast_div((uint32_t)rep);
    const PagedSeq q{0, rows, len};
    if (tr == 16) spans<16, 128>(a, q);
    else if (tr == 32) spans<32, 64>(a, q);
    else spans<128, 64>(a, q);
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("division")
    src = d / "spans.hip"
    src.write_text(PROGRAM)
    subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-host-only", "-c", str(src), "-o", str(d / "spans.o")], check=True,
                   capture_output=True)
    subprocess.run([build.HIPCC, str(d / "spans.o"), "-o", str(d / "spans")], check=True, capture_output=True)
    return str(d / "spans")


KEYS = {16: 128, 32: 64, 128: 64}


def expected(tr, rep, window, rows, len_):
    """[first, units] of each tile: from the tile of the first key that the tile's first row sees to that of its last row's own"""
    out = []
    for x0 in range(0, rows * rep, tr):
        x1 = min(rows * rep, x0 + tr)
        last = len_ - rows + (x1 - 1) // rep
        if last < 0:
            out += [0, 1]
            continue
        lo = max(0, len_ - rows + x0 // rep - window + 1) if window else 0
        out += [lo // KEYS[tr], last // KEYS[tr] - lo // KEYS[tr] + 1]
    return out


RAGGED = [(1, 1), (1, 200), (3, 3), (2, 129), (5, 2), (4, 0), (1, 64), (70, 300), (300, 7), (1000, 100000), (40, 2147482623),
          (20000, 0)]
TOP = 2 ** 31 - 1


def test_tiles_of_every_window(program):
    cases = [(tr, rep, w, rows, n) for tr in KEYS for rep in (1, 2, 7) for rows, n in RAGGED
             for w in (0, 1, 2, 17, 64, 100000, n - 1, n, n + 1, 2 ** 30, TOP - 1025, TOP - 1, TOP) if w >= 0]
    text = "\n".join(" ".join(map(str, c)) for c in cases)
    r = subprocess.run([program], input=text, capture_output=True, text=True, check=True, timeout=60)
    lines = r.stdout.splitlines()
    assert len(lines) == len(cases)
    for c, line in zip(cases, lines):
        assert [int(v) for v in line.split()] == expected(*c), c
