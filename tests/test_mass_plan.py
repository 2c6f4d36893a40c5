"""Which kernels a call of the drawn weight takes and how its keys are cut (``csrc/mass_plan.h``), compiled for the host: the calls that the GPU
tests make reach all of them, and pieces keep to what they are given."""
import subprocess

import pytest

from paper_2512_04939_amd import binding as B
from paper_2512_04939_amd import build

from mass_cases import CASES

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "mass_plan.h"
using namespace lv::mass;
// stdin: tokens, sequences, heads, kv heads, channels, type, room; rows' tokens and keys of each sequence.
// stdout: few scores keep own eight small splits, most pieces; then for the rows' sums and the keys': chunk, aim, and each sequence's pieces and chunks of a piece
int main() {
  int n, n_seq, heads, kv, dim, dtype;
  long long room;
  if (scanf("%d %d %d %d %d %d %lld", &n, &n_seq, &heads, &kv, &dim, &dtype, &room) != 7) return 1;
  std::vector<int> nq(n_seq), nk(n_seq);
  for (int i = 0; i < n_seq; ++i)
    if (scanf("%d %d", &nq[i], &nk[i]) != 2) return 1;
  const Form f = form_of(n, n_seq, heads, kv, dim, dtype, room);
  printf("%d %d %d %d %d %d %d %d\n", f.few, f.scores, f.keep, f.own, f.eight, f.small_chunks, f.splits, f.rows.most);
  for (const Cut &c : {f.rows, f.keys}) {
    const int group = heads / kv;
    float all = 0.f;
    for (int i = 0; i < n_seq; ++i) all += has_pieces(c, nq[i], nk[i]) ? chunk_cost(c, nq[i] * group) * (float)quotient_up(nk[i], c.chunk) : 0.f;
    const float work = piece_work(c, kv, all);
    printf("%d %d", c.chunk, c.aim);
    for (int i = 0; i < n_seq; ++i) {
      const bool any = has_pieces(c, nq[i], nk[i]);
      const int per = any ? chunks_of_piece(c, nq[i] * group, nk[i], work) : 0;
      printf(" %d %d", any ? quotient_up(quotient_up(nk[i], c.chunk), per) : 0, per);
    }
    printf("\n");
  }
}
"""
TYPES = dict(bf16=B.CACHE_BF16, e4m3=B.CACHE_E4M3, e2m1=B.CACHE_E2M1)


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("mass_plan")
    (d / "plan.hip").write_text(PROGRAM)
    subprocess.run(["hipcc", "-O1", "-std=c++17", "--offload-arch=gfx950", "-I", build.CSRC, str(d / "plan.hip"), "-o", str(d / "plan")],
                   check=True, capture_output=True)
    return str(d / "plan")


def plan(program, n, heads, kv_heads, head_dim, dtype, room, new, lens):
    text = f"{n} {len(new)} {heads} {kv_heads} {head_dim} {TYPES[dtype]} {room}\n" + "\n".join(f"{a} {b}" for a, b in zip(new, lens))
    r = subprocess.run([program], input=text, capture_output=True, text=True)
    assert r.returncode == 0
    lines = [[int(x) for x in line.split()] for line in r.stdout.splitlines()]
    form = dict(zip(("few", "scores", "keep", "own", "eight", "small", "splits", "most"), lines[0]))
    cuts = [dict(chunk=x[0], aim=x[1], pieces=x[2::2], per=x[3::2]) for x in lines[1:]]
    return form, *cuts


def words(f):
    if not f["few"]:
        return "many" + " small" * f["small"]
    return "few " + ("8" if f["eight"] else "32") + " kept" * f["keep"] + " own" * f["own"]


def planned(program, c, dtype):
    return plan(program, c["tokens"] or sum(c["new"]), c["heads"], c["kv_heads"], c["head_dim"], dtype, c["columns"] * c["page"], c["new"], c["lens"])


@pytest.mark.parametrize("c", CASES, ids=lambda c: c["name"])
def test_what_a_case_selects(program, c):
    for dtype in c["dtypes"]:
        form, by_rows, by_keys = planned(program, c, dtype)
        assert words(form) == c["form"], dtype
        assert (by_rows["per"][c["of"]], by_keys["per"][c["of"]]) == (c["rows_chunks"], c["keys_chunks"]), dtype


def test_the_cases_reach_everything(program):
    """Every kernel that a call may launch, for every type; pieces of several chunks in each of them where there are any; rows split and not."""
    seen, turns, splits = set(), set(), set()
    for c in CASES:
        for dtype in c["dtypes"]:
            form, by_rows, by_keys = planned(program, c, dtype)
            kind = (words(form).replace(" own", "").replace(" small", ""), c["head_dim"])
            seen |= {(dtype, "rows", *kind), (dtype, "keys", words(form), c["head_dim"])}
            if max(by_rows["per"]) > 1:
                turns.add(("rows", *kind))
            if max(by_keys["per"]) > 1:
                turns.add(("keys", words(form), c["head_dim"] if not form["keep"] else 0))
            if not form["few"]:
                splits.add(form["splits"] > 1)
    for dtype in TYPES:
        for dim in (64, 128):
            assert (dtype, "rows", "many", dim) in seen and (dtype, "keys", "many", dim) in seen
        assert (dtype, "rows", "few 8 kept", 64) in seen and (dtype, "rows", "few 32 kept", 64) in seen and (dtype, "keys", "few 8", 64) in seen
    assert ("e2m1", "keys", "few 32", 128) in seen and ("e4m3", "keys", "few 32", 128) in seen and ("bf16", "keys", "few 8", 128) in seen
    assert {("rows", "few 8 kept", 64), ("rows", "few 32 kept", 64), ("rows", "few 8", 64), ("rows", "few 32", 128), ("rows", "many", 64), ("rows", "many", 128),
            ("keys", "few 8 kept", 0), ("keys", "few 8", 64), ("keys", "few 32", 128), ("keys", "many", 64), ("keys", "many", 128),
            ("keys", "many small", 64)} <= turns
    assert splits == {False, True}


@pytest.mark.parametrize("heads,kv,dim,dtype", [(16, 16, 64, "e2m1"), (32, 4, 128, "bf16"), (1, 1, 64, "e4m3"), (1024, 1, 128, "e2m1")])
def test_pieces_keep_to_the_workspace(program, heads, kv, dim, dtype):
    """No more pieces of a sequence than its rows have room for, no more units than the grids have."""
    for room in (16, 5000, 1 << 20, 1 << 27):
        for new, lens in (([1], [room]), ([5, 5000, 0], [room, room // 2, room]), ([40] * 60, [room // (i + 1) for i in range(60)]),
                          ([1] * 300, [room] + [3] * 299), ([60000], [room])):
            n = sum(new)
            if n * heads >= 1 << 26:
                continue
            lens = [max(x, 1) for x in lens]
            form, *cuts = plan(program, n, heads, kv, dim, dtype, room, new, lens)
            rows = n * heads
            assert max(cuts[0]["pieces"]) <= form["most"] and form["most"] * rows <= max(1 << 25, rows)
            for c in cuts:
                pairs, chunks = len(new) * kv, -(-room // c["chunk"])
                assert sum(c["pieces"]) * kv <= min(c["aim"] + pairs, pairs * chunks)
                assert all(p * per >= -(-k // c["chunk"]) > (p - 1) * per for p, per, k, q in zip(c["pieces"], c["per"], lens, new) if p)
