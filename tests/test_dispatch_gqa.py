"""The form of the grouped-head attention against measured times (MI355X, 256 CUs),
and the sizes that follow from it: dispatch.h is compiled for the host."""
import math
import random

import pytest

from test_dispatch import CXX, _ask

pytestmark = pytest.mark.skipif(CXX is None, reason="no host C++ compiler")

# heads, kv heads, head dim, rows, requests, keys bound, causal prompt or pages; us of the whole call with 128 rows a
# workgroup, 128 with the keys cut, 32, 32 with the keys cut
BF16 = [
    (8, 8, 64, 1, 1, 8512, 0, 132.8, 25.8, 68.6, 25.0), (8, 8, 64, 7, 1, 2176, 0, 38.7, 18.1, 22.9, 18.4),
    (8, 8, 64, 47, 16, 256, 0, 10.2, 14.7, 8.7, 12.4), (8, 8, 64, 112, 1, 256, 0, 11.2, 11.5, 8.7, 11.4),
    (8, 8, 64, 186, 16, 256, 0, 10.6, 14.2, 8.6, 12.6), (8, 8, 64, 469, 16, 4032, 0, 67.3, 34.0, 38.1, 32.0),
    (8, 8, 64, 591, 4, 591, 1, 10.6, 13.9, 9.2, 14.1), (8, 8, 64, 1153, 1, 1153, 1, 20.5, 23.5, 15.0, 22.5),
    (8, 8, 64, 1498, 16, 320, 0, 12.7, 21.5, 11.1, 21.2), (14, 2, 64, 2, 2, 12032, 0, 183.3, 23.5, 92.7, 23.5),
    (14, 2, 64, 2, 2, 40064, 0, 604.7, 34.0, 299.0, 32.5), (14, 2, 64, 4, 4, 832, 0, 18.6, 12.7, 13.1, 12.4),
    (14, 2, 64, 12, 2, 12032, 0, 186.0, 23.1, 92.9, 23.9), (14, 2, 64, 16, 16, 20032, 0, 307.4, 37.5, 153.7, 36.3),
    (14, 2, 64, 39, 4, 39, 1, 8.9, 10.8, 8.1, 10.9), (14, 2, 64, 64, 64, 6016, 0, 97.5, 39.0, 51.9, 32.7),
    (14, 2, 64, 344, 4, 320, 0, 11.6, 14.6, 9.7, 15.0), (16, 1, 128, 2, 2, 12032, 0, 237.8, 23.9, 126.5, 24.6),
    (16, 1, 128, 4, 4, 2048, 0, 46.5, 16.0, 27.9, 15.9), (16, 1, 128, 16, 16, 2048, 0, 46.3, 20.1, 27.9, 17.5),
    (16, 1, 128, 469, 16, 256, 0, 14.1, 19.8, 11.1, 21.6), (16, 1, 128, 7876, 4, 7876, 1, 203.9, 179.8, 600.3, 466.1),
    (28, 4, 128, 1, 1, 3520, 0, 75.0, 23.2, 43.3, 23.8), (28, 4, 128, 1, 1, 11584, 0, 233.4, 28.1, 124.8, 27.9),
    (28, 4, 128, 7, 1, 2176, 0, 49.4, 19.5, 29.9, 20.7), (28, 4, 128, 56, 1, 2240, 0, 51.1, 32.2, 30.8, 23.7),
    (28, 4, 128, 64, 64, 448, 0, 17.2, 28.7, 13.5, 21.2), (28, 4, 128, 256, 256, 448, 0, 38.3, 50.5, 46.5, 41.4),
    (28, 4, 128, 877, 1, 3008, 0, 68.4, 59.8, 107.8, 114.2), (28, 4, 128, 897, 16, 897, 1, 12.1, 22.1, 30.9, 25.7),
    (28, 4, 128, 1498, 16, 1088, 0, 37.2, 50.1, 89.0, 75.7), (32, 8, 128, 1, 1, 8512, 0, 173.0, 30.4, 93.8, 29.3),
    (32, 8, 128, 4, 1, 192, 0, 10.5, 11.6, 10.0, 11.8), (32, 8, 128, 47, 16, 256, 0, 11.6, 17.6, 10.1, 13.6),
    (32, 8, 128, 77, 1, 77, 1, 9.8, 13.2, 9.5, 13.8), (32, 8, 128, 231, 1, 231, 1, 12.9, 21.9, 11.1, 22.3),
    (32, 8, 128, 1498, 16, 4096, 0, 113.0, 125.4, 236.6, 297.1), (32, 32, 128, 1, 1, 3520, 0, 76.3, 31.9, 44.1, 29.6),
    (32, 32, 128, 7, 1, 28352, 0, 583.1, 103.1, 311.7, 97.7), (32, 32, 128, 12, 2, 3008, 0, 65.7, 32.3, 39.8, 29.1),
    (32, 32, 128, 12, 2, 12032, 0, 250.8, 63.0, 138.1, 58.9), (32, 32, 128, 45, 8, 12032, 0, 277.1, 218.9, 211.5, 209.3),
    (32, 32, 128, 224, 1, 8768, 0, 182.5, 64.9, 105.9, 150.6), (32, 32, 128, 1075, 4, 4224, 0, 118.9, 100.8, 188.5, 252.9),
    (32, 32, 128, 1498, 16, 320, 0, 26.6, 44.6, 69.1, 54.9), (32, 32, 128, 2692, 16, 2692, 1, 34.1, 52.9, 98.2, 65.7),
    (32, 32, 128, 2954, 4, 2954, 1, 61.1, 79.5, 147.1, 150.5), (32, 32, 128, 5738, 8, 12544, 0, 1008.6, 1274.2, 2322.3, 3658.4),
]
# the same in fp32: uncut, cut
F32 = [
    (4, 4, 64, 7, 1, 64, 0, 9.1, 12.0), (4, 4, 64, 15, 1, 15, 1, 8.1, 11.1),
    (4, 4, 64, 16, 16, 2048, 0, 61.7, 23.5), (4, 4, 64, 64, 64, 256, 0, 11.5, 17.1),
    (4, 4, 64, 234, 16, 8064, 0, 226.5, 48.6), (6, 3, 32, 24, 4, 2048, 0, 38.0, 14.5),
    (6, 3, 32, 129, 4, 640, 0, 16.1, 13.0), (8, 1, 80, 51, 4, 8064, 0, 338.3, 33.5),
    (8, 1, 80, 406, 64, 2048, 0, 92.3, 48.8), (8, 1, 80, 880, 64, 64, 0, 11.5, 13.5),
    (8, 2, 128, 24, 4, 256, 0, 17.9, 13.7), (8, 2, 128, 64, 64, 8064, 0, 571.7, 154.6),
    (8, 2, 128, 77, 1, 77, 1, 12.7, 13.5), (8, 2, 128, 880, 64, 64, 0, 15.3, 16.9),
    (8, 2, 128, 8076, 16, 8076, 1, 253.5, 344.3), (32, 8, 128, 1, 1, 1216, 0, 53.6, 17.1),
]
RULE = """
static GqaLaunch launch(const long long* v) {
  return GqaLaunch{v[7] != 0, (int)v[0], (int)v[1], (int)v[2], (int)v[3], (int)v[4], v[5], v[6] != 0};
}
"""


def test_form(tmp_path):
    """The form taken is near the fastest on average, and never far from it."""
    rows = [r[:7] + (1,) for r in BF16] + [r[:7] + (0,) for r in F32]
    forms = _ask(tmp_path, RULE + "int answer(const long long* v) { GqaRule r = gqa_rule(launch(v)); return 2 * r.rt + r.cut; }",
                 rows)
    index = {256: 7, 257: 8, 64: 9, 65: 10, 32: 7, 33: 8}
    worst, total = 0.0, 0.0
    for r, f in zip(BF16 + F32, forms):
        lost = r[index[f]] / min(r[7:])
        worst, total = max(worst, lost), total + math.log(lost)
    assert worst <= 1.6 and total / len(forms) <= math.log(1.06), (worst, math.exp(total / len(forms)))


def test_what_follows_from_the_form(tmp_path):
    """Over random calls: the grid holds every tile of an uncut launch and no more parts than the workspace has room for;
    the places of a cut line fit 31 bits."""
    rng = random.Random(3)
    rows = []
    for _ in range(3000):
        kv = rng.choice([1, 2, 4, 8, 32])
        heads = kv * rng.choice([1, 2, 4, 7, 16, 71])
        bf16 = rng.random() < 0.7
        dim = rng.choice([64, 128]) if bf16 else rng.choice([4, 32, 64, 80, 128])
        n = int(math.exp(rng.uniform(0, math.log(2 ** 31 // heads - 1))))
        batch = int(math.exp(rng.uniform(0, math.log(5000))))
        rows.append((heads, kv, dim, n, batch, int(math.exp(rng.uniform(0, math.log(2 ** 31)))), rng.randint(0, 1), int(bf16)))
    body = RULE + """
int answer(const long long* v) {
  const GqaLaunch g = launch(v);
  const GqaRule r = gqa_rule(g);
  const long long pairs = (long long)g.rows * (g.heads / g.n_kv), tiles = gqa_tiles(g, r.rt);
  const long long lone = pairs >= g.batch ? (pairs - g.batch) / r.rt + g.batch : pairs;       // all rows but one a request in one
  if (tiles != lone * g.n_kv || r.grid < 1) return 1;
  if (!r.cut) return r.grid == tiles ? 0 : 2;
  if (r.grid > 1024 || r.grid > tiles * 32) return 3;
  if (tiles * ((g.keys + 63) / 64) > 0x7fffffff) return 4;
  return gqa_part_bytes(r.grid, r.rt, g.dim) <= gqa_workspace(g) ? 0 : 5;
}
"""
    assert set(_ask(tmp_path, body, rows)) == {0}


def test_division(tmp_path):
    """x / group by a multiplication, at the edges and between them."""
    rng = random.Random(4)
    rows = [(d, x) for d in list(range(1, 130)) + [255, 256, 257, 1000, 4095, 65535, 65536, 16777215, 2 ** 31 - 1]
            for x in [0, 1, d - 1, d, d + 1, 2 * d - 1, 2 ** 31 - 1, 2 ** 31 - 1 - (2 ** 31 - 1) % d, rng.randrange(2 ** 31)] if 0 <= x < 2 ** 31]
    body = """
int answer(const long long* v) {
  const GqaDivisor d = gqa_divisor((int)v[0]);
  const unsigned x = (unsigned)v[1];
  return (int)(((unsigned)((unsigned long long)x * d.mul >> 32) + x) >> d.shift);
}
"""
    assert _ask(tmp_path, body, rows) == [x // d for d, x in rows]
