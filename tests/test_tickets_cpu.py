"""Ticket words in memory of any contents: every order in which workgroups can draw, on the host."""
import os
import subprocess

import pytest

from paper_2412_03213_amd.build import CSRC, CXX

MODEL = r"""
#include <stdio.h>
#include <stdlib.h>
#include "ticket.hpp"
using ck::Ticket;
typedef Ticket::Word Word;

// One workgroup draws in atomic steps: a fetch-add, then compare-and-swaps where what was there is none of ours,
// and the store of the last one.
enum { BEFORE, SWAP, LAST, DONE };
struct Group { int at; Word seen; };
struct State { Word w; Group g[3]; };

static int N;
static long runs;

static void fail(Word start, const char* what) {
  printf("%016llx, %d arrivals: %s\n", start, N, what);
  exit(1);
}
static void drawn(State& s, int i, Word now, Word start) {
  s.g[i].at = Ticket::complete(now, N) ? LAST : DONE;
  if (s.g[i].at == LAST)
    for (int j = 0; j < N; ++j)
      if (j != i && s.g[j].at != DONE) fail(start, "one is the last before all have arrived");
}
static void explore(const State& s, Word start) {
  bool more = false;
  for (int i = 0; i < N; ++i) {
    if (s.g[i].at == DONE) continue;
    more = true;
    State t = s;
    if (s.g[i].at == BEFORE) {
      t.w = s.w + Ticket::ONE;
      if (Ticket::count(s.w, N) >= 0) {
        drawn(t, i, t.w, start);
      } else {
        t.g[i].at = SWAP;
        t.g[i].seen = t.w;
      }
    } else if (s.g[i].at == SWAP) {
      if (s.w == s.g[i].seen) {
        t.w = Ticket::after(s.w, N);
        drawn(t, i, t.w, start);
      } else {
        t.g[i].seen = s.w;
      }
    } else {
      t.w = Ticket::IDLE;
      t.g[i].at = DONE;
    }
    explore(t, start);
  }
  if (more) return;
  ++runs;
  if (s.w != Ticket::IDLE) fail(start, "not idle afterwards: nobody was the last");
}

int main() {
  const Word I = Ticket::IDLE, O = Ticket::ONE;
  const Word values[] = {1, 2, 3, 4, 0x80, 0xFF, 0x3F80, 0x4B43, 0x5469, 0x636B, 0x8000, 0xFFFF};
  for (N = 1; N <= 3; ++N) {
    auto from = [](Word w) { explore(State{w, {}}, w); };
    from(I);
    const Word others[] = {0ull, ~0ull, 1ull, 0x434B5061676E0001ull, 0x434B7469636B0001ull, I - 1, I - O, I - 2 * O,
                           I - 3 * O, I + 0xFFFF * O, I + N * O, I + (N + 1) * O};
    for (Word w : others)
      from(w);
    for (int keep = 0; keep < 15; ++keep)               // 16-bit parts of an idle word that are overwritten
      for (Word v : values) {
        Word w = I;
        for (int p = 0; p < 4; ++p)
          if (!(keep >> p & 1)) w = (w & ~(0xFFFFull << 16 * p)) | v << 16 * p;
        from(w);
      }
    for (int byte = 0; byte < 8; ++byte)
      for (Word v = 0; v < 256; ++v) from((I & ~(0xFFull << 8 * byte)) | v << 8 * byte);
  }
  printf("%ld orders\n", runs);
  return 0;
}
"""


def test_every_order_of_arrivals_has_one_last(tmp_path):
    src, exe = tmp_path / "model.cpp", tmp_path / "model"
    src.write_text(MODEL)
    subprocess.run([CXX, "-O2", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout.split()[0]) > 1000
