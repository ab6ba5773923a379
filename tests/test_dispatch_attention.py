"""Workgroups of differential attention (csrc/agc_dispatch.h), compiled with the host compiler: launches of fewer than 2^32
threads over the whole documented range, every tile of every key head met once.  CPU only."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

DRIVER = r"""
#include "agc_dispatch.h"
extern "C" int columns(int causal, int n_seqs, int kv_heads, int slots, int splits)
{
    return agc::attn_columns(causal != 0, n_seqs, kv_heads, slots, splits);
}
extern "C" int blocks(int columns, int n_seqs, int kv_heads, int slots, int splits)
{
    return agc::attn_blocks(columns, n_seqs, kv_heads, slots, splits);
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("attention")
    (tmp / "driver.cpp").write_text(DRIVER)
    cxx = shutil.which("g++") or shutil.which("c++")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fPIC", "-shared",
                    "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-I", os.path.join(ROOT, "paper_2605_15890_amd", "csrc"), str(tmp / "driver.cpp"),
                    "-o", str(tmp / "librules.so")], check=True)
    return ctypes.CDLL(str(tmp / "librules.so"))


@pytest.mark.parametrize("kv_heads", [1, 2, 3, 4, 5, 8, 16, 24, 64, 1024, 65536])
@pytest.mark.parametrize("causal", [0, 1])
def test_fewer_threads_than_a_launch_takes(rules, kv_heads, causal):
    """Rows of all key heads up to 2^30, sequences times key heads up to 2^21; a large workgroup has 256 rows and 512 threads, and
    2^21 rows of G may lie behind the keys' pass."""
    for log_seqs in range(21):
        n_seqs = min(1 << log_seqs, (1 << 21) // kv_heads)
        for rows in (256, 1000, 2048, 1 << 14, (1 << 30) // kv_heads // max(n_seqs, 1)):
            if n_seqs == 0 or rows < 256 or rows * n_seqs * kv_heads > 1 << 30:
                continue
            slots = rows * n_seqs // 256 + n_seqs
            columns = rules.columns(causal, n_seqs, kv_heads, slots, 1)
            blocks = rules.blocks(columns, n_seqs, kv_heads, slots, 1)
            assert slots * kv_heads <= blocks and ((blocks + 7) // 8 * 8 + (1 << 21) - 1) * 512 < 1 << 32, (n_seqs, rows)


@pytest.mark.parametrize("n_seqs,kv_heads,slots", [(8, 16, 72), (4, 4, 132), (1, 8, 64), (5, 1, 600), (3, 2, 301), (7, 24, 100)])
def test_columns_meet_every_tile_once(rules, n_seqs, kv_heads, slots):
    columns = rules.columns(1, n_seqs, kv_heads, slots, 1)
    assert columns == -(-slots // n_seqs)
    met = []
    share, rows = max(8 // kv_heads, 1), max(kv_heads // 8, 1) * n_seqs
    for wg in range(rules.blocks(columns, n_seqs, kv_heads, slots, 1)):
        x, i = wg & 7, wg >> 3
        step, row = divmod(i, rows)
        head, seq = divmod(row, n_seqs)
        column = step * share + x % share
        slot = seq * columns + column
        if column < columns and slot < slots:
            met.append((x * (kv_heads // 8) + head if kv_heads >= 8 else x // share, slot))
    assert sorted(met) == [(h, s) for h in range(kv_heads) for s in range(slots)]


def test_what_takes_no_columns(rules):
    assert rules.columns(0, 8, 16, 72, 1) == 0 and rules.columns(1, 8, 16, 72, 2) == 0      # no mask, splits
    assert rules.columns(1, 8, 3, 400, 1) == 0 and rules.columns(1, 8, 12, 400, 1) == 0     # heads that do not go round the XCDs
    assert rules.columns(1, 8, 16, 31, 1) == 0                                             # too few tiles
