"""The products' rings of stages, as product_ring.h orders them for the kernels, followed load
by load in a host build (CPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_21290_amd", "csrc")
CXX = shutil.which("g++") or shutil.which("c++")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <map>
#include <utility>
#include "product_ring.h"

#define MUST(what) \
  do { if (!(what)) { std::printf("%s: down %d %d, loads %d %d, halves %d .. %d\n", #what, DA, DB, LA, LB, h0, h1); std::exit(1); } } while (0)

// One wave's loads in order, what each place of the two rings holds, and how far its reads are.
template <bool DA, bool DB, int LA, int LB>
void follow(int h0, int h1) {
  constexpr uint32_t PA = 4096, PB = 6144;
  using Ring = gl::ProductRing<DA, DB, LA, LB, PA, PB>;
  static_assert(Ring::after_even >= 0 && Ring::after_even < 64 && Ring::after_odd >= 0 && Ring::after_odd < 64, "six bits");
  struct Place { int piece, end; int last_read; };  // piece, its loads' number, the wait count of its last read
  std::map<std::pair<int, uint32_t>, Place> places;
  int issued = 0, landed = 0, waits = 0, reading = h0, multiplied = h0, held[2] = {-1, -1};
  const bool down[2] = {DA, DB};
  auto load = [&](int op, int piece, uint32_t at) {
    const uint32_t bytes = op ? PB : PA;
    const int ring = op ? Ring::RB : Ring::RA, loads = op ? LB : LA;
    MUST(at % bytes == 0 && at / bytes < (uint32_t)ring);
    MUST(piece >= (down[op] ? h0 : h0 / 2) && (down[op] ? piece : 2 * piece) < h1);
    auto old = places.find({op, at});
    if (old != places.end()) {
      // every half of what lay there has been read, and a barrier has passed since
      const int last = down[op] ? old->second.piece : 2 * old->second.piece + 1;
      MUST(last < reading && old->second.last_read < waits);
    }
    issued += loads;
    places[{op, at}] = {piece, issued, 1 << 30};
  };
  auto wait_for = [&](int n) {
    ++waits;
    if (issued - n > landed) landed = issued - n;
  };
  Ring::run(
      h0, h1, [&](int piece, uint32_t at) { load(0, piece, at); }, [&](int piece, uint32_t at) { load(1, piece, at); },
      [&](auto n) { wait_for(decltype(n)::value); }, [&] { wait_for(0); },
      [&](auto set, uint32_t a, uint32_t b) {
        MUST(reading % 2 == decltype(set)::value);
        if (reading < h1)  // (one read more, of whatever lies there, ends the contraction)
          for (int op = 0; op < 2; ++op) {
            auto p = places.find({op, op ? b : a});
            MUST(p != places.end());
            MUST(p->second.piece == (down[op] ? reading : reading / 2));
            MUST(p->second.end <= landed);
            p->second.last_read = waits;
          }
        else
          MUST(reading == h1 && a / PA < (uint32_t)Ring::RA && b / PB < (uint32_t)Ring::RB);
        held[decltype(set)::value] = reading++;
      },
      [&](auto set) {
        MUST(held[decltype(set)::value] == multiplied);
        ++multiplied;
      });
  MUST(multiplied == h1);    // every half once
  MUST(landed == issued);    // none under way when the epilogue writes LDS
  long long all = 0;         // and every piece loaded once
  for (int op = 0; op < 2; ++op) all += (long long)(down[op] ? h1 - h0 : (h1 - h0) / 2) * (op ? LB : LA);
  MUST(issued == all);
}

template <bool DA, bool DB, int LA, int LB>
void all() {
  for (int stages = 0; stages < 40; ++stages)
    for (int first : {0, 1, 2, 5, 8}) follow<DA, DB, LA, LB>(2 * first, 2 * (first + stages));
}

int main() {
  // loads a piece of the tiles of 256, 128, 64 and 32: the same for both operands, twice as
  // many for whole stages; and other ratios
  all<false, false, 4, 4>(); all<false, false, 2, 2>(); all<false, false, 1, 1>(); all<false, false, 8, 8>();
  all<false, true, 4, 2>(); all<false, true, 8, 4>(); all<false, true, 2, 1>(); all<false, true, 1, 4>();
  all<true, false, 2, 4>(); all<true, false, 4, 1>();
  all<true, true, 2, 2>(); all<true, true, 4, 4>(); all<true, true, 1, 1>(); all<true, true, 1, 4>();
  return 0;
}
"""


def _run(tmp_path, header):
    (tmp_path / "product_ring.h").write_text(header)
    src, exe = tmp_path / "ring.cpp", tmp_path / "ring"
    src.write_text(PROGRAM)
    subprocess.run([CXX, "-std=c++17", "-I", str(tmp_path), str(src), "-o", str(exe)], check=True, capture_output=True)
    return subprocess.run([str(exe)], capture_output=True, text=True)


def _header():
    with open(os.path.join(CSRC, "product_ring.h")) as f:
        return f.read()


@pytest.mark.skipif(CXX is None, reason="no host compiler")
def test_a_ring_is_read_after_it_has_landed_and_filled_after_it_was_read(tmp_path):
    r = _run(tmp_path, _header())
    assert r.returncode == 0, r.stdout


@pytest.mark.skipif(CXX is None, reason="no host compiler")
@pytest.mark.parametrize("old,new", [
    ("by_half_even = (rh - 2)", "by_half_even = (rh - 1)"),
    ("by_stage = (rs - 2) * per_stage", "by_stage = (rs - 1) * per_stage"),
    ("by_half_odd < by_stage ? by_half_odd : by_stage", "by_half_odd < by_stage ? by_stage : by_half_odd"),
    ("if (HA && h + RA < h1) load_a(h + RA, pa);", "if (HA && h + RA < h1) load_a(h + RA, next(pa, PA, RA));"),
    ("2 * ((h >> 1) + RB) < h1) load_b", "2 * ((h >> 1) + RB) <= h1) load_b"),
    ("        fill(h, false);\n", ""),
    ("LAST = 2 * (RA > RB ? RA : RB);", "LAST = 0;"),
])
def test_a_planted_mistake_is_found(tmp_path, old, new):
    text = _header()
    assert old in text
    r = _run(tmp_path, text.replace(old, new, 1))
    assert r.returncode != 0, (old, new)


def test_the_kernels_take_their_order_from_it():
    with open(os.path.join(CSRC, "product.h")) as f:
        text = f.read()
    assert "ProductRing<G::KA, G::KB," in text and "Ring::run(" in text and "product_ring_depth(KA, KB)" in text
    assert text.count("la.load(") == 1 and text.count("lb.load(") == 1
