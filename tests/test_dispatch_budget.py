"""The rules of attention weights and eviction (CPU): dispatch.h is compiled for the host."""
import math
import random

import pytest

from test_dispatch import CXX, _ask

pytestmark = pytest.mark.skipif(CXX is None, reason="no host C++ compiler")


def _spread(rng, most):
    return int(math.exp(rng.uniform(0, math.log(most))))


def test_workspace_of_weights(tmp_path):
    """A call that stays within the rows and requests of a larger one fits its workspace: its parts' statistics
    (rows, heads, parts) and its scores (rows, heads, places)."""
    rng = random.Random(5)
    rows = []
    for _ in range(4000):
        kv = rng.choice([1, 2, 4, 8, 32])
        heads = kv * rng.choice([1, 2, 4, 7, 16, 71])
        most = _spread(rng, 2 ** 30 // heads - 1)
        batch = _spread(rng, 4096)
        n, b = (most, batch) if rng.random() < 0.3 else (_spread(rng, most), _spread(rng, batch))
        rows.append((n, b, most, batch, heads, kv, 16 * _spread(rng, 2 ** 20), rng.randint(0, 1)))
    body = """
int answer(const long long* v) {
  const int b = (int)v[1], batch = (int)v[3], heads = (int)v[4], kv = (int)v[5];
  const long long places = v[6];
  const bool bf16 = v[7];
  const bool few = weights_few(v[0], b, heads, kv, places, bf16);
  const int parts = weights_parts(v[0], b, heads, kv, places, bf16, few);
  if (parts < 1 || parts > kWeightsParts) return 1;
  if (v[0] * heads * parts > weights_stats(v[2], heads, bf16)) return 2;
  if (few && v[0] * heads * places > weights_scores(v[2], batch, heads, kv, places, bf16)) return 3;
  if (few && !bf16) return 4;
  const int sums = weights_sums(v[0], b, heads, kv, places);
  if (sums < 1 || sums > kWeightsSums || (sums > 1 && sums * (long long)b * kv * places > kWeightsPartial)) return 6;
  return weights_scores(v[2], batch, heads, kv, places, bf16) > kWeightsScores ? 5 : 0;
}
"""
    assert set(_ask(tmp_path, body, rows)) == {0}


def test_form_of_weights(tmp_path):
    """Scores are kept where a request has few rows, and not where they would be many."""
    rows = [(1, 1, 32, 8, 4096, 1), (64, 64, 32, 8, 4096, 1), (1, 1, 32, 8, 4096, 0), (64, 4, 32, 8, 4096, 1),
            (16, 4, 32, 8, 4096, 1), (17, 4, 32, 8, 4096, 1), (64, 64, 32, 8, 1 << 20, 1), (1, 1, 16, 1, 1 << 20, 1)]
    body = """int answer(const long long* v) { return weights_few(v[0], (int)v[1], (int)v[2], (int)v[3], v[4], v[5]); }"""
    assert _ask(tmp_path, body, rows) == [1, 1, 0, 0, 1, 0, 0, 1]


def test_eviction(tmp_path):
    """A list fits the kernel that is chosen for it; the workgroup that moves its own rows has room for their slots in LDS;
    a list's slots and bits fit its part of the workspace."""
    rng = random.Random(6)
    rows = [(l, s, n) for l in (1, 255, 256, 511, 512, 4096, 2 ** 20 - 1) for s in (0, 1)
            for n in (16, 2048, 2064, 8192, 8208, 16384, 16400, 2 ** 20)]
    rows += [(_spread(rng, 2 ** 20), rng.randint(0, 1), 16 * _spread(rng, 2 ** 17)) for _ in range(500)]
    body = """
int answer(const long long* v) {
  const EvictRule r = evict_rule((int)v[0], v[1], v[2]);
  if (r.places && r.places < v[2]) return 1;
  if (!r.places && v[2] <= 16384) return 2;
  if (r.fused && (v[1] || r.places != 2048)) return 3;
  if (r.parts < 1 || r.parts * v[0] >= 1ll << 24) return 4;
  if (2 * evict_room(v[2]) < (size_t)v[2] || evict_room(v[2]) % 64) return 5;
  // slots from and to, then a bit of each place in whole words
  const size_t words = (v[2] + 63) / 64;
  return evict_list_bytes(v[2]) < 8 * evict_room(v[2]) + 8 * words ? 6 : 0;
}
"""
    assert set(_ask(tmp_path, body, rows)) == {0}
