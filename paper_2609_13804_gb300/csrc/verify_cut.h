// How the rows of a verification are cut, and the most parts that a call of no more rows and logits can have.  Plain C++ on the
// host, too.
#pragma once
#include <algorithm>
#include <cstddef>

namespace sp {

constexpr int kRowSlices = 32;  // of a row, at most

struct Cut {
  int slices;
  bool ordered;
};

inline int most_slices(int V) { return std::max(1, std::min(kRowSlices, (V + 2047) / 2048)); }
inline int wave_slices(int V) { return std::min(most_slices(V), (V + 51199) / 51200); }  // of a row of a call of many waves

// slots: CTAs of the sums that run at once.  Rows that fit one wave of them are cut into as many slices as do (of at least
// 2,048 logits), more into slices of about 51,200.  In order, with decisions on the way, where several rows of a sequence can be
// passed over and they are more than is soon read (64 sequences of 8 drafts, 152,064 bf16 logits: 72 us in order, 77 not; of 5
// drafts, 96 of 50,001 fp32: 56, 52; 200 of 3, 5,000 fp32: 26, 21).
inline Cut verify_cut(int T_cap, int B, int V, int max_rows, bool drafted, bool f32, int slots) {
  const int rows = std::max(drafted ? 2 * T_cap - std::min(B, T_cap) : T_cap, 1);
  Cut c;
  c.ordered = rows > slots && max_rows > 3 && (double)rows * V * (f32 ? 4 : 2) > 0x1p28;
  c.slices = rows > slots ? wave_slices(V) : std::max(1, std::min(most_slices(V), (slots + rows / 2) / rows));
  return c;
}

// T_cap * slices of any call of up to T_cap rows of up to V logits: as many as rows have slices at most; and in one wave, with
// rows >= T_cap of them, T_cap (slots / rows + 1 / 2) <= slots + slots / 2.  Grows with T_cap and V, so a workspace for the largest
// step serves smaller ones, which are cut into more slices.
inline size_t verify_parts(int T_cap, int V, int slots) {
  const size_t T = (size_t)T_cap, wave = (size_t)slots + slots / 2;
  return std::min(T * most_slices(V), std::max(wave, T * wave_slices(V)));
}

}  // namespace sp
