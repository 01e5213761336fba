"""The words that kernels of routed calls report to: a report by work of a route that is gone does not reach the next owner of its word."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cassert>
#include <cstdlib>
#include "gm_route_words.h"
using namespace gm;

static int slabs = 0;
static void* more(size_t bytes) { ++slabs; return std::malloc(bytes); }
static void* none(size_t) { return nullptr; }

int main() {
  RouteWords words;
  assert(!words.take(none).at);
  // a report reaches its own route, until the route is given back
  RouteWord a = words.take(more);
  assert(!route_word_reported(a));
  route_word_report(a);
  assert(route_word_reported(a));
  words.give(a);
  // the word's next owner begins without one; the old owner's late kernel (or its graph's replay) changes nothing for it
  RouteWord b = words.take(more);
  assert(b.at == a.at && !route_word_reported(b));
  route_word_report(a);
  assert(!route_word_reported(b));
  // nor does it take away the new owner's own report
  route_word_report(b);
  route_word_report(a);
  assert(route_word_reported(b));
  words.give(b);
  // the same after the numbers have wrapped around
  RouteWord last{b.at, 0xffffffffu};
  words.give(last);
  RouteWord c = words.take(more);
  assert(c.owner == 0 && !route_word_reported(c));
  route_word_report(last);
  assert(!route_word_reported(c));
  route_word_report(c);
  route_word_report(last);
  assert(route_word_reported(c));
  // routes that live at the same time have words of their own, from as many slabs as it takes
  RouteWord many[3000];
  for (RouteWord& w : many) { w = words.take(more); assert(w.at && !route_word_reported(w)); }
  route_word_report(many[1234]);
  for (int i = 0; i < 3000; ++i) assert(route_word_reported(many[i]) == (i == 1234));
  assert(slabs == 3);
  for (RouteWord& w : many) words.give(w);
  for (RouteWord& w : many) { w = words.take(more); assert(!route_word_reported(w)); }
  assert(slabs == 3);
  words.give(RouteWord{});
  return 0;
}
"""


def test_reports_stay_with_their_owner(tmp_path):
    source, program = tmp_path / "words.cpp", tmp_path / "words"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "paper_2607_22866_b200", "csrc"), "-o", str(program), str(source)], check=True)
    subprocess.run([str(program)], check=True, timeout=60)
