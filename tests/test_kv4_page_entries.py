"""Which entries of a page table the attention's tiles read, compiled for the host: for every tile of both kernels that begins before a
sequence's end, the entry that holds its tokens, and none behind the sequence's last."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2101_05615_amd", "csrc")

SHIM = r"""
#include "qg_pages.h"
// Tiles of 32 tokens in stages of one or two, as the kernels walk them; entries read that the sequence does not have, or that are not
// the page of a token it has
extern "C" long long bad_entries(int keys, int lgp, int stage) {
  const int entries = qg_page_entries(keys, lgp);
  long long bad = entries != (keys + (1 << lgp) - 1) / (1 << lgp);
  for (int t0 = 0; t0 < keys; t0 += stage)
    for (int t = t0; t < t0 + stage; t += 32)
      for (int half = 0; half < 2; ++half) {
        const int e = qg_page_entry(t, half, lgp, entries), token = t + 16 * half;
        bad += e < 0 || e >= entries || (token < keys && e != token / (1 << lgp));
      }
  return bad;
}
"""


@pytest.fixture(scope="module")
def bad_entries(tmp_path_factory):
    d = tmp_path_factory.mktemp("pages")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "shim.cpp"), "-o", str(d / "shim.so")], check=True)
    f = ctypes.CDLL(str(d / "shim.so")).bad_entries
    f.argtypes, f.restype = [ctypes.c_int] * 3, ctypes.c_longlong
    return f


@pytest.mark.parametrize("stage", [32, 64])
@pytest.mark.parametrize("lgp", [4, 5, 6, 7, 8])
def test_entries(bad_entries, lgp, stage):
    for keys in list(range(1, 1200)) + [131071, 131072, 131073, (1 << 30) - 1 >> 6]:
        assert bad_entries(keys, lgp, stage) == 0, keys


def test_the_kernels_read_through_it():
    """One place reads the page table, by that function and with the sequence's own number of entries."""
    text = open(os.path.join(CSRC, "qg_kv4_tile.h")).read()
    assert text.count("table[") == 1 and "table[qg_page_entry(t0, half, lgp, entries)]" in text and "qg_page_entries(keys, p.c.lgp)" in text
    for name in ("kv4_attention.hip", "kv4_attention_rows.hip"):
        text = open(os.path.join(CSRC, name)).read()
        assert "in(p, j.seq, j.keys, j.head, r, g);" in text and "p.pages" not in text
