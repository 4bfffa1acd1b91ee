// The rows of a scan's sequences (csrc/dgc_steps.h) for offsets of every kind, in arithmetic of 128 bits.
#include "dgc_steps.h"

#include <cstdio>
#include <initializer_list>

int main() {
  const int64_t least = INT64_MIN, most = INT64_MAX, mega = (int64_t)1 << 40;
  const int64_t offsets[] = {least, least + 1, least / 2, -mega, -5, -1, 0, 1, 2, 19, 20, 21, 99, 100, 101, mega - 1, mega, most / 2, most - 1, most};
  long checked = 0;
  for (int64_t rows : {(int64_t)0, (int64_t)1, (int64_t)100, mega - 1})
    for (int64_t longest : {(int64_t)0, (int64_t)1, (int64_t)20, (int64_t)1 << 31})
      for (int64_t lo : offsets)
        for (int64_t hi : offsets) {
          const dgc::SequenceRows got(lo, hi, rows, longest);
          __int128 begin = lo, end = hi;
          begin = begin < 0 ? 0 : begin > rows ? rows : begin;
          end = end > rows ? (__int128)rows : end;
          __int128 length = end - begin;
          length = length < 0 ? 0 : length > longest ? (__int128)longest : length;
          if (got.begin != begin || got.length != length || got.begin < 0 || got.length < 0 || got.begin + got.length > rows) {
            std::printf("offsets %lld, %lld, %lld rows, %lld at most: %lld and %lld\n", (long long)lo, (long long)hi, (long long)rows,
                        (long long)longest, (long long)got.begin, (long long)got.length);
            return 1;
          }
          ++checked;
        }
  std::printf("ok %ld sequences\n", checked);
  return 0;
}
