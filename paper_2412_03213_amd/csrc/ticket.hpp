// Ticket words: how the workgroups that leave partial results find out which of them is the last, in
// memory of any contents.
//
// A word holds a mark between two copies of the number of arrivals, the upper one moved by a constant.  Arriving adds one
// to both.  A word whose copies do not agree, whose mark is another, or whose count is one that the call does not
// leave, is none of ours: memory that was never used, or an idle word of which something was overwritten
// since, be it a byte, one of the copies, or both with the same value.  The first arrival takes its place.
#pragma once
#include <stdint.h>

namespace ck {

struct Ticket {
  typedef unsigned long long Word;
  static constexpr Word ONE = (1ull << 48) | 1ull;
  static constexpr Word IDLE = 0x4B435469636B0000ull;   // no arrival: 0x5469636B between 0x4B43 and 0
  // arrivals that a word stands for, of fewer than `expected`; -1: none of ours
  static constexpr int count(Word w, int expected) {
    const Word k = w & 0xFFFFull;
    return w == IDLE + (k << 48 | k) && (int)k < expected ? (int)k : -1;
  }
  // what an arrival that has not been counted yet makes of a word
  static constexpr Word after(Word w, int expected) { return (count(w, expected) < 0 ? IDLE : w) + ONE; }
  static constexpr bool complete(Word w, int expected) { return w == IDLE + (Word)expected * ONE; }
};

}  // namespace ck
