// Prints how the tiles of a shared-prefix call are dealt out: tiles of a worker, the multiple that units are counted as, 1 if waves
// are the workers, what the units count for.  Command line: workgroups, then "units:tiles" for units alike.
#include <cstdio>
#include <cstdlib>

#include "../../paper_2603_04428_amd/csrc/prefix_plan.h"

int main(int argc, char **argv)
{
    auto counted = [&](int round) -> long long { // of one layer and KV head: the kernel adds them up in int
        int sum = 0;
        for (int i = 2; i < argc; ++i) {
            char *at;
            const int units = (int)strtol(argv[i], &at, 10), tiles = (int)strtol(at + 1, nullptr, 10);
            sum += units * q4kv::rounded_up(tiles, round);
        }
        return sum;
    };
    long long units = 0;
    for (int i = 2; i < argc; ++i) units += strtoll(argv[i], nullptr, 10);
    int per = 0, round = 0;
    const bool solo = q4kv::spread((int)counted(1), (int)units, atoi(argv[1]), per, round, counted);
    printf("%d %d %d %lld\n", per, round, solo ? 1 : 0, counted(round));
    return 0;
}
