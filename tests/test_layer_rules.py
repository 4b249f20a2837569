"""Every kernel that the rules by size of the layers by role, in 8-bit integers and from kept bytes choose is run by a size of the GPU
tests: a rule that changes takes no kernel out of them unseen. The rules are host code (csrc/rules.h), compiled here."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

import layer_forms
import test_gpu_grouped
import test_gpu_int8
import test_gpu_packed
from paper_2606_12950_amd import _layers

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_12950_amd", "csrc")

# What a call launches, as words. A weights' gradient: its tile, s for shares across the groups, g for units by group, 1 where no second
# launch follows, + where only groups of two units have places in the workspace. Operators are called with the input's gradient (x) and without.
SOURCE = r"""
#include "rules.h"
#include <string>
using namespace maestro;
typedef std::string S;
static S text(int64_t v) { return std::to_string(v); }
static S tile(int64_t p, int64_t q) { return text(p) + "x" + text(q); }
static S grouped(int64_t n, int64_t groups, int64_t i, int64_t o, bool bf16, bool x) {
  const bool pair = bf16 ? grouped_bf16::paired(grouped_bf16::cut_of(n, groups, i, o), n, i) : grouped_f32::paired(grouped_f32::cut_of(n, i, o), n, i);
  S out, cut;
  int64_t k;
  bool by_group;
  if (bf16) {
    const auto c = grouped_bf16::cut_of(n, groups, i, o);
    k = c.k_split, by_group = c.by_group, cut = tile(c.tp, c.tq);
    out = "y" + text(grouped_bf16::tile_of(false, o, n));
    if (x && !pair) out += " gx" + text(grouped_bf16::tile_of(true, i, n));
  } else {
    const auto c = grouped_f32::cut_of(n, i, o);
    k = c.k_split, by_group = c.by_group, cut = c.wide ? "128" : "64";
    out = grouped_f32::wide_forward(o, n, i) ? "y128" : "y64";
    if (x && !pair) out += grouped_f32::wide(i, n) ? " gx128" : " gx64";
  }
  const S way = S(by_group ? "g" : "s") + (n <= k ? "1" : shared_places(n, groups, k) ? "+" : "");
  out += S(x && pair ? " pair" : " gw") + cut + way;
  if (n > k) out += " join" + way + (grouped_f32::join_dealt(n, groups, k, i * o, o) ? "16" : "");
  return out;
}
static S packed(int64_t n, int64_t i, int64_t o, bool bf16, bool x) {
  if (bf16) {
    const auto c = packed_bf16::cut_of(n, i, o);
    const int t = packed_bf16::tile_of(i, n);
    const S cut = tile(c.tp, c.tq) + (c.splits == 1 ? "1" : "");
    return !x ? "gw" + cut : t == 64 ? "pair" + cut : "gx" + text(t) + " gw" + cut;
  }
  const auto c = packed_f32::cut_of(n, i, o);
  const S cut = S(c.wide ? "128" : "64") + (c.splits == 1 ? "1" : "");
  return !x ? "gw" + cut : packed_f32::paired(c, n, i) ? "pair" + cut : S(packed_f32::wide(i, n) ? "gx128" : "gx64") + " gw" + cut;
}
static S quantised(int64_t n, int64_t i, int64_t o) {
  const auto l = int8::row_lanes((int32_t)i);
  const auto t = int8::product_tile(o, n);
  return "rows" + text(l.units) + " y" + tile(t.tile, t.wavefronts);
}
extern "C" int64_t place(int64_t group, int64_t row, int64_t per) { return first_place((int)group, (int)row, (int)per); }
extern "C" int64_t places(int64_t n, int64_t groups, int64_t per) { return places_of(n, groups, per); }
extern "C" int shared(int64_t n, int64_t groups, int64_t per) { return shared_places(n, groups, per); }
extern "C" void form(int op, int64_t n, int64_t groups, int64_t i, int64_t o, int bf16, int x, char* out, size_t size) {
  const S s = op == 0 ? grouped(n, groups, i, o, bf16, x) : op == 1 ? packed(n, i, o, bf16, x) : quantised(n, i, o);
  s.copy(out, size - 1);
  out[s.size() < size ? s.size() : size - 1] = 0;
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    source, lib = str(d / "forms.cpp"), str(d / "forms.so")
    open(source, "w").write(SOURCE)
    compiler = os.environ.get("CXX") or shutil.which("g++") or "/opt/rocm/bin/amdclang++"
    subprocess.run([compiler, "-O1", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror", f"-I{CSRC}", source, "-o", lib], check=True)
    return ctypes.CDLL(lib)


@pytest.fixture(scope="module")
def forms(rules):
    call = rules.form
    call.argtypes = [ctypes.c_int, *[ctypes.c_int64] * 4, ctypes.c_int, ctypes.c_int, ctypes.c_char_p, ctypes.c_size_t]
    call.restype = None
    text = ctypes.create_string_buffer(256)

    def of(op, n, groups, i, o, bf16, x):
        call(op, n, groups, i, o, bf16, x, text, 256)
        return text.value.decode().split()
    return of


def sizes_of(test):
    """The sizes that a test is parametrized with."""
    return [tuple(v) for m in test.pytestmark if m.name == "parametrize" and m.args[0].endswith("i,o") for v in m.args[1]]


TESTED = {
    0: [(sum(s), len(s), i, o) for t in (test_gpu_grouped.test_groups, test_gpu_grouped.test_many_rows) for s, i, o in sizes_of(t)] +
       [(sum(s) + 8, len(s), i, o) for s, i, o in layer_forms.GROUPED],
    1: [(n, 1, i, o) for n, i, o in sizes_of(test_gpu_packed.test_layer_grad_packed) + layer_forms.PACKED],
    2: [(n, 1, i, o) for n, i, o in sizes_of(test_gpu_int8.test_layer_int8) + layer_forms.INT8] +
       [(n, 1, d, 16) for t in [test_gpu_int8.test_quantize_rows] for n, d in test_gpu_int8.SHAPES],
}


@pytest.mark.parametrize("op", [0, 1, 2])
@pytest.mark.parametrize("bf16", [0, 1])
def test_every_form_is_tested(forms, op, bf16):
    x = (0, 1) if op < 2 else (0,)
    tested = {f for n, g, i, o in TESTED[op] for w in x for f in forms(op, n, g, i, o, bf16, w)}
    r = random.Random(op)
    chosen = {}
    span = lambda most: int(round(most ** r.random()))
    for _ in range(60000):
        n, g, i, o = span(1 << 27), span(256) if op == 0 else 1, 16 * span(1024), 16 * span(1024)
        for f in forms(op, n, g, i, o, bf16, r.choice(x)):
            chosen.setdefault(f, (n, g, i, o))
    assert not {f: chosen[f] for f in chosen if f not in tested}


def test_forms_that_no_size_chooses(forms):
    """The launchers have no kernel for these: bfloat16 gradients of kept bytes in one launch beside 256-wide tiles of the weights', and
    256 x 256 tiles of the groups' weights' gradient by group, 64 x 64 ones by shares; nor,
    where only groups of two units have places, 128 x 128 float32 ones by group and a join of few values' shares."""
    r = random.Random(7)
    span = lambda low, most: int(round(low * (most / low) ** r.random()))
    for _ in range(60000):
        n, i, o = span(1, 1 << 28), 16 * span(1, 1024), 16 * span(1, 1024)
        narrow = 16 * r.randint(1, 4)                         # 256 x 64 tiles' outputs
        assert not {f for f in (*forms(1, n, 1, i, o, 1, 1), *forms(1, n, 1, i, narrow, 1, 1)) if f.startswith("pair256")}, (n, i, o, narrow)
        groups, few = span(1, 256), 16 * span(1, 16)
        none = ("gw256x256g", "gw64x64s", "gw128g+", "joins+16")
        for bf16 in (0, 1):
            assert not {f for f in (*forms(0, n, groups, i, o, bf16, 0), *forms(0, n, 256, few, narrow, bf16, 0)) if f.startswith(none)}, (n, groups, i, o)
    # at the edges of both rules: the least rows that leave a 64-wide tile, and the most that stay in one
    for i in range(144, 16385, 16):
        for o in (16, 48, 64):
            for n in {k + d for k in (128 * 255 // -(-i // 128), 128 * 256 // -(-i // 128), 512, 131072) for d in range(-2, 131)} - {0}:
                assert not {f for f in forms(1, max(n, 1), 1, i, o, 1, 1) if f.startswith("pair256")}, (n, i, o)


@pytest.mark.parametrize("by_group", [False, True])
def test_places_of_shares(rules, by_group):
    """Every unit of the groups that have two or more has a place of its own, below the count that sizes the workspace: numbered as units come,
    and where groups are many from a group's first_place on."""
    for f in (rules.place, rules.places):
        f.argtypes, f.restype = [ctypes.c_int64] * 3, ctypes.c_int64
    rules.shared.argtypes = [ctypes.c_int64] * 3
    r, seen = random.Random(3), set()
    for _ in range(6000):
        groups, per = r.choice([1, 2, 3, 8, 40, 256]), r.choice([1, 2, 5, 64])
        choice = r.choice([[0, 1, per - 1, per, per + 1, 2 * per, 2 * per + 1, r.randint(0, 7 * per)], [per + 1, 2, 2 * per], [0, 0, 0, 0, 0, 0, 1, 2, per + 1]])
        sizes = [r.choice(choice) for _ in range(groups)]
        n = sum(sizes) + r.choice([0, 0, 1, per])                  # rows of no group
        if n <= per:
            continue                                               # no group has two units
        few, most = bool(rules.shared(n, groups, per)), rules.places(n, groups, per)
        seen.add(few)
        taken, row, before = set(), 0, 0
        for g, size in enumerate(sizes):
            units = -(-size // per) if by_group else ((row + size - 1) // per - row // per + 1 if size else 0)
            if units > 1:
                first = rules.place(g, row, per) if few else before
                assert first >= 0 and not taken & set(range(first, first + units)), (sizes, per, g)
                taken |= set(range(first, first + units))
            row += size
            before += units
        assert max(taken, default=-1) < most <= 3 * (n // per), (sizes, per)
    assert seen == {False, True}


def test_workspace_of_many_groups():
    """Groups of few rows write their gradients themselves: the workspace has at most three places for each unit that the rows fill, however
    many the groups are."""
    ws = _layers.load().maestro_layer_grouped_grad_workspace
    for n, i, o in ((4096, 1024, 1024), (8000, 2048, 2048), (20000, 1024, 1024), (40000, 512, 768), (300, 2048, 2048)):
        for bf16, least in ((0, 128), (1, 512)):              # rows of a unit: no fewer, but for the last multiple of 64
            for groups in (1, 16, 64, 256):
                need = ws(n, groups, i, o, bf16)
                assert need <= 3 * (n // (least - 64)) * 4 * (i + 1) * o, (n, groups, i, o, bf16, need)
                assert need <= (n // (least - 64) + groups) * 4 * (i + 1) * o
    assert ws(20000, 256, 1024, 1024, 1) <= 64 << 20
    assert ws(4096, 256, 1024, 1024, 1) <= 80 << 20
