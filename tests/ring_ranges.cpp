// Every copy that the rounds of layer norm's rows off 16-byte boundaries make, as the kernels make them, within the
// matrix but for bytes that share 16 with it?  Prints the copies, and those that leave it.
#include <cstdio>

#include "tula_ring.h"

int main() {
    long copies = 0, outside = 0;
    const int kN = 16, kMostThreads = 512;
    const int widths[] = {1, 2, 3, 4, 5, 6, 7, 8, 9, 15, 16, 17, 31, 33, 100, 250, 257, 1001, 4097, 8191};
    for (int size = 2; size <= 4; size += 2)
        for (int cols : widths) {
            int group = 1;
            while (group < kMostThreads && group * kN < cols) group *= 2;
            const int per = (group > 256 ? group : 256) / group, bytes = cols * size;
            for (int more = 0; more < 9; ++more)          // elements between the rows
                for (int start = 0; start < 16; start += size)  // the first one's place in its 16 bytes
                    for (int over = 0; over < 4; ++over)
                        for (int full = 1; full < 4; ++full) {
                            const long long rows = (long long)full * per + over, stride = cols + more;
                            const long long end = start + ((rows - 1) * stride + cols) * size;
                            for (long long r0 = 0; r0 < rows; r0 += per) {
                                if (r0 == 0 || r0 > tula::last_round_copied(rows, per, bytes)) continue;
                                const long long n = rows - r0 < per ? rows - r0 : per;
                                auto check = [&](long long at, int length) {
                                    const unsigned off = (unsigned)(at & 15);
                                    const long long from = at - off, to = from + tula::bytes_copied(off, length);
                                    ++copies;
                                    outside += from < start || to > end || to < at + length;
                                };
                                if (more == 0)
                                    check(start + r0 * stride * size, (int)n * bytes);
                                else
                                    for (long long g = 0; g < n; ++g) check(start + (r0 + g) * stride * size, bytes);
                            }
                        }
        }
    std::printf("%ld %ld\n", copies, outside);
    return 0;
}
