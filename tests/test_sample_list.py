"""How many tokens a segment of a row puts into its list, on the host: the rule that the kernel goes by
(paper_2511_20340_amd/csrc/sample_rules.h), fed with the kernel's counts, which numpy repeats in float32.  Whatever the
logits are, the list has room for what is taken, and it is whole down to where it says."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SEG, BINS, ROOM, OFF = 8192, 256, 512, 2 ** 31 - 1
SOURCE = """
#include "sample_rules.h"
static_assert(sf::SAMPLE_BINS == 256 && sf::SAMPLE_ROOM == 512, "sizes");
extern "C" int depth(const int *counts, int bounded, int top_bucket, int bound_bucket, int k) {
  const int whole = sf::sample_whole_bins(bounded, top_bucket, bound_bucket);
  int upto = 0;
  for (int b = 0; b < sf::SAMPLE_BINS; ++b) {
    upto += counts[b];
    if (!sf::sample_takes(b, counts[b], upto, whole, k)) return b;
  }
  return sf::SAMPLE_BINS;
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    (d / "rule.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2511_20340_amd", "csrc"),
                    "-o", str(d / "rule.so"), str(d / "rule.cpp")], check=True)
    L = C.CDLL(str(d / "rule.so"))
    L.depth.argtypes = [np.ctypeslib.ndpointer(np.int32), C.c_int, C.c_int, C.c_int, C.c_int]
    return L


def buckets(l, g):
    with np.errstate(over="ignore"):
        return np.floor(np.maximum(l * np.float32(g), np.float32(-131072))).astype(np.int64)


def listed(rule, logits, temperature, k):
    """(bins taken, tokens that go into the list) of one segment for a count of k (OFF: a least weight alone)."""
    l = np.full(SEG, np.nan, np.float32)
    l[:len(logits)] = logits
    g = 8.0 / float(np.clip(np.float32(temperature), 1, 2))
    # thread t holds tokens 4 t .. 4 t + 3 of every 1024; NaN never wins
    own = np.fmax.reduce(np.concatenate([l.reshape(8, 256, 4).transpose(1, 0, 2).reshape(256, 32), np.full((256, 1), -np.inf, np.float32)], 1), 1)
    top, bound = own.max(), own.min()
    if OFF > k > 256:
        bound = np.float32(-np.inf)
    if not abs(float(top) * g) < 65536:
        return 0, 0                                         # off the grid: no list
    first = int(buckets(top, g))
    there = l > -np.inf
    counted = there & (l >= bound)
    rel = np.minimum(first - buckets(l[counted], g), BINS - 1)
    counts = np.bincount(rel, minlength=BINS).astype(np.int32)
    bounded = bound > -np.inf
    deep = rule.depth(counts, int(bounded), first, int(buckets(bound, g)) if bounded else 0, k)
    if deep >= BINS:
        return deep, int(there.sum())
    return deep, int((there & (buckets(np.where(there, l, -np.inf), g) > first - deep)).sum())


def crowd(every, low, lead, base=0.0):
    x = np.full(SEG, low, np.float32)
    x[::every] = base
    x[5] = lead
    return x


@pytest.mark.parametrize("k", [1, 2, 20, 50, 256, OFF])
@pytest.mark.parametrize("every", [2, 16, 17, 18, 20, 26, 28, 30, 32, 33])
def test_a_lead_over_a_patterned_crowd(rule, every, k):
    for low in (-1.0, -50.0, -1e4, float(np.finfo(np.float32).min)):
        for lead in (5.0, 31.0, 31.9, 32.0, 40.0, 100.0, 8000.0):
            for t in (0.5, 1.0, 1.3, 2.0, 9.0):
                deep, n = listed(rule, crowd(every, low, lead), t, k)
                assert n <= ROOM, (low, lead, t, deep, n)


@pytest.mark.parametrize("k", [20, 50, 256, OFF])
def test_one_allowed_token_for_each_thread(rule, k):
    rng = np.random.default_rng(k % 1000)
    for low in (-50.0, -1e4):
        x = np.full(SEG, low, np.float32)
        x[np.arange(256) * 4 + rng.integers(0, 4, 256) + 1024 * rng.integers(0, 8, 256)] = rng.normal(size=256)
        for lead in (20.0, 32.0, 40.0, 64.5, 100.0):
            y = x.copy()
            y[77] = lead
            for t in (1.0, 1.7, 2.0):
                deep, n = listed(rule, y, t, k)
                assert n <= ROOM, (low, lead, t, deep, n)


def test_random_rows(rule):
    rng = np.random.default_rng(1)
    for it in range(400):
        n = int(rng.choice([1, 5, 255, 256, 1024, 5000, SEG]))
        x = rng.normal(size=n) * 10.0 ** rng.uniform(-3, 3)
        if it % 3 == 0:
            x[np.arange(n) % int(rng.integers(2, 40)) != 0] -= 10.0 ** rng.uniform(0, 4)
        if it % 4 == 1:
            x[rng.random(n) < 0.5] = rng.choice([-np.inf, np.nan])
        x[int(rng.integers(n))] = rng.uniform(0, 100)
        for k in (1, 50, 256, 257, 1000, OFF):
            deep, taken = listed(rule, x.astype(np.float32), float(rng.choice([0.7, 1.0, 1.5, 3.0])), k)
            assert taken <= ROOM, (it, k, deep, taken)
