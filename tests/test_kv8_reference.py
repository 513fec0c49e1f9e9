"""CPU: the plain 8-bit cache of the tests, and the cache's block numbers as the
kernels compute them."""
import itertools
import os
import subprocess

import numpy as np
import pytest

import kv8
from helpers import ROOT
from paper_2608_10139_gb300 import build


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_a_tile_holds_every_element_once(hd):
    k, v = kv8.tile_maps(hd)
    at = np.concatenate([k.ravel(), v.ravel()])
    assert sorted(at) == list(range(64 * hd))
    assert (k < 32 * hd).all() and (v >= 32 * hd).all()
    # a block's first keys are a prefix of both halves, in steps of 16
    assert (k[:16] < 16 * hd).all() and (v[:16] < 48 * hd).all()
    if hd > 32:
        for n in (8, 16, 24):
            assert (k[:n] < n * hd).all()


def test_values_are_within_half_a_step():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((32, 64)).astype(np.float16)
    q, s = kv8.quantize(x)
    assert np.abs(q).max() == 127
    assert (np.abs(q * np.float64(s) - x) <= np.float64(s) / 2 * (1 + 1e-6)).all()
    assert kv8.quantize(np.zeros((32, 64), np.float16))[1] == 0
    q, _ = kv8.quantize(np.array([[127, 63.5, -63.5, 0.5, -0.5, 0.4995]], np.float16))
    assert q.tolist() == [[127, 64, -64, 1, -1, 0]]


PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "tile8.cuh"
using namespace aiq;
int main() {
  unsigned x = 12345;
  for (int trial = 0; trial < 20000; ++trial) {
    x = x * 1664525u + 1013904223u;
    const int n = 1 + (x >> 20) % 9;
    int64_t start = 0, next = 0;
    for (int r = 0; r < n; ++r) {
      x = x * 1664525u + 1013904223u;
      const int64_t len = (x >> 18) % 100;
      const int64_t first = tile8_first_block(start, r);
      if (first < next) return printf("sequence %d begins inside the one before\n", r), 1;
      next = first + (len + kTileKeys - 1) / kTileKeys;
      start += len;
    }
    if (next > tile8_blocks(start, n)) return printf("more blocks than promised\n"), 1;
  }
  return 0;
}
"""


def test_blocks_of_sequences_do_not_meet(tmp_path):
    src, exe = tmp_path / "blocks.cu", tmp_path / "blocks"
    src.write_text(PROGRAM)
    r = subprocess.run([build.nvcc()] + build.ARCH + build.FLAGS + [str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""})
    assert r.returncode == 0, r.stdout


def test_blocks_of_every_small_batch():
    for lens in itertools.product([0, 1, 31, 32, 33, 63, 64], repeat=4):
        st, end = kv8.starts(lens), 0
        for r, n in enumerate(lens):
            b = kv8.first_block(int(st[r]), r)
            assert b >= end
            end = b - (-n // 32)
        assert end <= kv8.blocks(sum(lens), len(lens))


def test_sample_by_hand():
    z = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    order = [1, 3, 2, 0]
    for u, want in ((0.0, 0), (0.39, 0), (0.41, 1), (0.69, 1), (0.71, 2), (0.89, 2), (0.91, 3)):
        assert kv8.sample(z, u, 1.0, 4, 1.0, 0.0)[0] == order[want]
    assert kv8.sample(z, 0.99, 1.0, 2, 1.0, 0.0)[0] == 3          # top-k
    assert kv8.sample(z, 0.99, 1.0, 4, 0.65, 0.0)[0] == 3         # top-p: 0.4 + 0.3
    assert kv8.sample(z, 0.99, 1.0, 4, 1.0, 0.45)[0] == 2         # min-p: 0.2 / 0.4 is in, 0.1 / 0.4 is not
    assert abs(kv8.sample(z, 0.99, 1.0, 4, 1.0, 0.45)[1] - 0.2 / 0.9) < 1e-12
    assert kv8.sample(np.zeros(4), 0.5, 1.0, 4, 0.5, 0.0)[0] == 1  # equal logits: two are kept
