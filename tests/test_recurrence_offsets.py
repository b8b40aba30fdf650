"""Where the gated recurrence's words and carried states lie, on the host: rows times channels past 2^31.  (The kernels' own function, compiled for the CPU; a call of this size holds 50 GB.)"""
import ctypes
import glob
import os
import re
import subprocess

import numpy as np
import pytest

import __graft_entry__ as entry

ROOT = os.path.dirname(os.path.abspath(entry.__file__))
CSRC = os.path.join(ROOT, "paper_2605_21325_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "gated_recurrence.cuh"
int main() {
  long long begin, index, D, c;
  int seq, tile;
  while (std::scanf("%lld %d %d %lld %lld %lld", &begin, &seq, &tile, &index, &D, &c) == 6) {
    const int slot = (int)(tri_inv::rec_slot(begin, seq, tile) + index);   // an int, as it lies in a block's ring of tiles
    std::printf("%lld\n", tri_inv::rec_at(slot, (int)D, (int)c));
  }
}
"""


def cases():
    """(first token, sequence, tokens of a tile, tile, channels, channel): 524288 sequences of one token, then a long one, and the ends of what a call may have."""
    for tile in (64, 128):
        for n in (0, 1, 524288, 600000):
            for D, c in ((1, 0), (4096, 0), (4096, 4095), (5000, 4999), (2 ** 26, 2 ** 26 - 1)):
                yield n, n, tile, 4, D, c
        yield 2 ** 31 - 129, 2 ** 24, tile, 1, 2048, 7


def test_rows_times_channels_pass_32_bits(tmp_path):
    source, program = tmp_path / "offsets.cu", tmp_path / "offsets"
    source.write_text(PROGRAM)
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                           str(source), "-o", str(program)])
    given = list(cases())
    got = subprocess.run([str(program)], input="\n".join(" ".join(map(str, x)) for x in given), capture_output=True, text=True, check=True).stdout.split()
    want = [(n // tile + seq + index) * D + c for n, seq, tile, index, D, c in given]
    assert [int(x) for x in got] == want
    assert max(want) > 2 ** 40 and sum(2 ** 31 <= x < 2 ** 33 for x in want) > 4


def test_the_kernels_form_no_such_place_themselves():
    for path in glob.glob(os.path.join(CSRC, "gated_recurrence*kernel.cu")):
        for line in open(path):
            assert not re.search(r"(slot|seq|index)[^;]*\* a\.D\b", re.sub(r"\(long long\)[^;]*", "", line)), (path, line)


@pytest.mark.parametrize("dtype", [0, 1])
def test_the_workspace_holds_the_last_word(dtype):
    entry.build()
    from paper_2605_21325_b200 import binding as b
    lens, D = [1] * 524288 + [300], 4096
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    need, rows = ctypes.c_size_t(0), ctypes.c_int64(0)
    desc = b.RecDesc(1, int(cu[-1]), D, (b.F32, b.BF16)[dtype], b.REC_GATE, len(lens), cu.ctypes.data)
    assert b.load().tri_inv_gated_recurrence_backward_workspace(desc, 1, need) == b.OK and b.load().tri_inv_gated_recurrence_carries(desc, rows) == b.OK
    tile = 64 if dtype == 0 else 128
    last = 524288 // tile + 524288 + (300 - 1) // tile
    assert last * D > 2 ** 31 and need.value >= 8 * (last + 1) * D
    assert rows.value > 524288 // 64 + 524288 + 299 // 64 - 1
