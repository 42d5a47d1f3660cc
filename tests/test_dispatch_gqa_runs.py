"""Which cut lines of the grouped-head attention are laid in runs (dispatch.h, compiled for the host): never with a run
of no length, however many tiles a call has."""
import random

import pytest

from test_dispatch import CXX, _ask
from test_dispatch_gqa import RULE

pytestmark = pytest.mark.skipif(CXX is None, reason="no host C++ compiler")

BODY = RULE + """
int answer(const long long* v) {
  const GqaLaunch g = launch(v);
  const GqaRule r = gqa_rule(g);
  if (!r.cut) return 0;
  const long long tiles = gqa_tiles(g, r.rt), line = tiles * ((g.keys + 63) / 64);
  for (int most = r.grid; most > 0; most = most > 256 ? 256 : 0)
    for (int part = 0; part < 4; ++part) {              // lines up to the longest that the bounds allow
      const int all = (int)(part == 0 ? line : line * part / 4);
      const bool runs = gqa_in_runs(all, most, (int)tiles);
      if (runs != (all > most && tiles > 1 && 2 * tiles <= most)) return 1;
      if (runs && gqa_run_room(all, most, (int)tiles) < 1) return 2;
    }
  return 3;
}
"""


def test_two_to_the_thirty_tiles(tmp_path):
    """2^20 rows in as many requests, 1024 heads on 1024: cut, and far too many tiles for runs."""
    assert _ask(tmp_path, BODY, [(1024, 1024, 4, 1 << 20, 1 << 20, 16, 0, 0), (1024, 1024, 4, 1 << 20, 1 << 20, 64, 0, 0)]) == [3, 3]


def test_over_the_range(tmp_path):
    rng = random.Random(7)
    rows = []
    for _ in range(4000):
        bf16 = rng.random() < 0.6
        kv = int(2 ** rng.uniform(0, 12))
        heads = kv * rng.choice([1, 1, 2, 7, 71])
        n = int(2 ** rng.uniform(0, 31)) // heads or 1
        batch = int(2 ** rng.uniform(0, 24))
        rows.append((heads, kv, rng.choice([64, 128]) if bf16 else rng.choice([4, 64, 80, 128]), n, batch,
                     int(2 ** rng.uniform(0, 31)), rng.randint(0, 1), int(bf16)))
    got = _ask(tmp_path, BODY, rows)
    assert set(got) <= {0, 3} and got.count(3) > 500


def test_keys_of_a_request(tmp_path):
    """No more than the table has, and four tiles behind the last key an int still holds their places."""
    rows = [(n, w, s) for n in (-5, 0, 1, 63, 4096, 2 ** 30, 2 ** 31 - 1025, 2 ** 31 - 1024, 2 ** 31 - 1)
            for w in (1, 10, 2 ** 23, 2 ** 31 - 1) for s in (4, 6, 8)]
    got = _ask(tmp_path, "int answer(const long long* v) { return gqa_keys((int)v[0], (int)v[1], (int)v[2]); }", rows)
    assert got == [max(0, min(n, w << s, 2 ** 31 - 1024)) for n, w, s in rows]
