"""The arithmetic by which attention over keys of another set gives its workgroups their work (``csrc/kv_plan.h``), compiled for the host
and run over sequences' shares, from offsets that ascend and from ones that do not."""
import os
import subprocess

import pytest

from paper_2512_04939_amd import build

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include <algorithm>
#include "kv_plan.h"
// stdin: room for units, room for slots, sequences, then units and slots of each; the plan as the kernel makes it, 1024 sequences at a time in
// waves of 64.  stdout: starts, slots before each, then for every unit of the grid: sequence, its number in it, whether it is there.
int main() {
  int room, slots, n;
  if (scanf("%d %d %d", &room, &slots, &n) != 3) return 1;
  std::vector<int> units(n), taken(n), starts(n), before(n);
  for (int i = 0; i < n; ++i)
    if (scanf("%d %d", &units[i], &taken[i]) != 2) return 1;
  int b[2] = {0, 0};
  const int rooms[2] = {room, slots};
  const std::vector<int> *own[2] = {&units, &taken};
  std::vector<int> *out[2] = {&starts, &before};
  for (int what = 0; what < 2; ++what)
    for (int chunk = 0; chunk < n; chunk += 1024) {
      int at = 0;
      for (int wave = chunk; wave < chunk + 1024; wave += 64) {
        int sum = 0;
        for (int i = wave; i < std::min(wave + 64, n); ++i) {
          (*out[what])[i] = lv::start_of(b[what], at + sum, rooms[what]);
          if (__builtin_add_overflow(sum, lv::share_of((*own[what])[i], rooms[what]), &sum)) return 2;
        }
        if (__builtin_add_overflow(at, lv::share_of(sum, rooms[what]), &at)) return 2;
      }
      b[what] = lv::start_of(b[what], at, rooms[what]);
    }
  for (int i = 0; i < n; ++i) printf("%d %d\n", starts[i], before[i]);
  for (int u = 0; u < room; u += std::max(1, room / 20000)) {
    const int s = (int)(std::upper_bound(starts.begin(), starts.end(), u) - starts.begin()) - 1;
    const int local = u - starts[s];
    printf("%d %d %d\n", s, local, (int)lv::unit_there(local, units[s], taken[s] > 0, local + before[s], slots));
  }
}
"""


KEYS = r"""
#include <cstdio>
#include <cmath>
#include "kv_plan.h"
// the candidate with the least key, of 64 whose costs come on stdin
int main() {
  float cost;
  uint32_t least = 0xffffffffu;
  for (int i = 0; i < 64; ++i) {
    if (scanf("%f", &cost) != 1) return 1;
    const uint32_t key = lv::cost_key(cost, i);
    least = key < least ? key : least;
  }
  printf("%d\n", lv::candidate_of(least));
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv_plan")
    (d / "plan.hip").write_text(PROGRAM)
    subprocess.run(["hipcc", "-O1", "-std=c++17", "--offload-arch=gfx950", "-I", build.CSRC, str(d / "plan.hip"), "-o", str(d / "plan")],
                   check=True, capture_output=True)
    return str(d / "plan")


def plan(program, room, slots, units, taken):
    text = f"{room} {slots} {len(units)}\n" + "\n".join(f"{u} {t}" for u, t in zip(units, taken))
    r = subprocess.run([program], input=text, capture_output=True, text=True)
    assert r.returncode == 0
    lines = [[int(x) for x in line.split()] for line in r.stdout.splitlines()]
    return [x[0] for x in lines[:len(units)]], [x[1] for x in lines[:len(units)]], lines[len(units):]


def test_units_of_offsets_that_ascend(program):
    units = [3, 0, 0, 7, 1, 12, 0] * 400
    taken = [0, 0, 0, 7, 0, 12, 0] * 400
    room, slots = sum(units) + 5, sum(taken)
    starts, before, found = plan(program, room, slots, units, taken)
    at = [0, 0]
    owner = []
    for s, (u, t) in enumerate(zip(units, taken)):
        assert [starts[s], before[s]] == at
        owner += [(s, i) for i in range(u)]
        at = [at[0] + u, at[1] + t]
    assert [(s, i) for s, i, there in found if there] == owner
    assert not any(there for _, _, there in found[len(owner):])


@pytest.mark.parametrize("n_seq,kv_heads,n_q", [(54210, 64, 1048575), (65535, 64, 1048000), (65, 1, 1 << 24), (4096, 1024, 65535)])
@pytest.mark.parametrize("cut", [False, True])
def test_units_of_offsets_that_do_not_ascend(program, n_seq, kv_heads, n_q, cut):
    """Every other sequence claims nearly all rows: the sum is far beyond 2^31 (or the room), and whatever is found is a unit of its sequence,
    and a slot of the workspace."""
    n_q -= n_q % 2
    units = [(n_q - s) * kv_heads // 32 if s % 2 == 0 else 0 for s in range(n_seq)]
    room = (n_q // 32 + n_seq) * kv_heads + 1536
    slots = 3000 if cut else 0
    taken = units if cut else [0] * n_seq
    starts, before, found = plan(program, room, slots, units, taken)
    assert max(units) * (n_seq // 2) > room and starts == sorted(starts) and before == sorted(before)
    assert 0 <= starts[0] and starts[-1] <= room and 0 <= before[0] and before[-1] <= slots
    for s, local, there in found:
        assert local >= 0
        assert not there or (local < units[s] and (not taken[s] or 0 <= local + before[s] < slots))


def test_numbers_below_zero_are_no_units(program):
    """What a wrapped sum gave: local = -2076502332 of 12788 blocks times 64 heads.  (Starts that fall would have to be made up: the plan has none.)"""
    source = PROGRAM[:PROGRAM.index("int main")] + r"""
int main() {
  const int units = 12788 * 64;
  return lv::unit_there(-2076502332, units, false, 0, 0) || lv::unit_there(-1, units, false, 0, 0) || lv::unit_there(0, units, true, -1, 3000) ||
         lv::unit_there(units, units, false, 0, 0) || lv::unit_there(0, 0, false, 0, 0) || !lv::unit_there(units - 1, units, false, -1, 0) ||
         !lv::unit_there(0, units, true, 2999, 3000) || lv::unit_there(0, units, true, 3000, 3000);
}
"""
    d = os.path.dirname(program)
    with open(os.path.join(d, "below.hip"), "w") as f:
        f.write(source)
    subprocess.run(["hipcc", "-O1", "-std=c++17", "--offload-arch=gfx950", "-I", build.CSRC, os.path.join(d, "below.hip"), "-o", os.path.join(d, "below")],
                   check=True, capture_output=True)
    assert subprocess.run([os.path.join(d, "below")]).returncode == 0


def test_the_least_cost_is_chosen_however_large_the_costs_are(program):
    """Up to 2^27 (262,144 blocks of 256 rows over 2^24 keys: 512 rounds of 262,144 tiles) and beyond; of equal ones the last."""
    d = os.path.dirname(program)
    with open(os.path.join(d, "keys.hip"), "w") as f:
        f.write(KEYS)
    subprocess.run(["hipcc", "-O1", "-std=c++17", "--offload-arch=gfx950", "-I", build.CSRC, os.path.join(d, "keys.hip"), "-o", os.path.join(d, "keys")],
                   check=True, capture_output=True)

    def chosen(costs):
        r = subprocess.run([os.path.join(d, "keys")], input=" ".join(str(c) for c in costs), capture_output=True, text=True)
        return int(r.stdout)

    for size in (0, 7, 100, 1 << 17, 1 << 23, (1 << 23) + 8, 1 << 27, 1 << 31, 1 << 40):
        for best in (0, 20, 62, 63):
            costs = [size + max(size // 50, 1) * (1 + i % 9) for i in range(64)]
            costs[best] = size
            assert chosen(costs) == best, (size, best)
        assert chosen([size] * 64) == 63 and chosen([size] * 30 + [2 * size + 1] * 34) == 29
