// The decode kernel's addresses of keys, for every lane: prints the largest end of a load past its key's end, and loads that are not of their key's own words.
#include <cstdio>

#include "vq_attention.hpp"

int main() {
  long long past = 0, other = 0;
  for (int bytes = 1; bytes <= 2; ++bytes)
    for (int dim = 16; dim <= 256; dim += 16)
      for (int shift = 4; shift <= 8; ++shift)
        for (int head = 0; head < 2; ++head)
          for (int place = 0; place < 512; place += 16)
            for (int lane = 0; lane < 64; ++lane)
              for (int t = 0; t < 4; ++t)
                for (int w = 0; w < (dim + 63) / 64 * 64 * bytes / 64; ++w) {
                  const int n = lane & 15, g = lane >> 4, row = dim * bytes;
                  const long long key = ((long long)head << shift) + place % (1 << shift) + 4 * t + n % 4;
                  const long long at = vq::key_word_at(head, shift, place, t, w, n, g, row);
                  if (at < key * row) past = 1 << 20;
                  if (at + 16 - (key + 1) * row > past) past = at + 16 - (key + 1) * row;
                  other += w * 64 + g * 16 < row && at != key * row + w * 64 + g * 16;
                }
  printf("%lld %lld\n", past, other);
  return 0;
}
