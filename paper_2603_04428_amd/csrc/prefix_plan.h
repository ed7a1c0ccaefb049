// How the tiles of a shared-prefix call are dealt out to its waves: arithmetic on counts alone, in a header of its own so that it can be
// checked without a GPU (every workgroup does it for itself, on the device).
#pragma once
#ifdef __HIP__
#define Q4KV_PLAN __host__ __device__ __forceinline__
#else
#define Q4KV_PLAN inline
#endif

namespace q4kv {

constexpr int kPlanWaves = 4;         // of a workgroup
constexpr int kSoloTiles = 2;         // smallest range of a wave on its own
constexpr int kPart = 3, kJoin = 1;   // in tiles' time: see spread()
constexpr int kJoinBelow = 16;        // tiles per wave from which workgroups are not considered
constexpr int kMostTiles = 0x7fffffff; // places in the plan are int, those of units counted as longer than they are too

// n / d for 0 <= n < 2^31, 0 < d and a quotient below 2^21: the product with the reciprocal errs by less than one
Q4KV_PLAN int quotient(int n, int d)
{
#ifdef __HIP_DEVICE_COMPILE__
    int q = (int)((float)n * __builtin_amdgcn_rcpf((float)d));
    const int r = n - q * d;
    q += r < 0 ? -1 : (r >= d ? 1 : 0);
    return q;
#else
    return n / d;
#endif
}

// (v below 2^21 * round)
Q4KV_PLAN int rounded_up(int v, int round) { return round == 1 ? v : quotient(v + round - 1, round) * round; }

Q4KV_PLAN int larger(int a, int b) { return a > b ? a : b; }

// `per` tiles a worker, units counted as the next multiple of `round`; true: the waves are the workers, else the workgroups,
// whose waves take a range tile by tile in turn.  `total`: tiles of the call, `units`: units that have any, padded(r): the tiles with
// every unit's rounded up to r.
// A worker pays for every part of a unit it begins (block ids, first tiles, queries: kPart tiles' time), so units are
// cut into ranges of their own that are equally long but for each unit's last, if there are workers enough for them all and the
// ranges are not much longer for it.  A workgroup as a worker joins its waves' sums in LDS (kJoin tiles' time) and leaves one
// record instead of four.  Else every wave takes an equal range wherever it begins.  Measured (us; only workgroups or, from 16 tiles a
// wave on, waves with ranges anywhere / as here): 128-wide, ten agents behind 4,096, four layers 50.2 / 37.9; 64-wide, 14 behind 5,376,
// eleven layers 47.0 / 29.7; 192 + 128, eight behind 2,048, three layers 38.8 / 27.9; 256-wide, 40 behind 1,024 46.4 / 35.3, ten behind
// 8,192 27.9 / 27.8.  Ranges of their own whatever their length: 32 agents of 128-wide heads behind 16,384, two layers 82 -> 104.
template <typename F>
Q4KV_PLAN bool spread(int total, int units, int workgroups, int &per, int &round, F padded)
{
    auto fit = [&](int workers, int step) { // the shortest range, a multiple of `step`; 0: none
        if (units > workers) return 0;
        int r = rounded_up(quotient(total, workers - units / 2) + 1, step); // a unit's last range is half empty, about
#pragma unroll 1
        for (int k = 0; k < 4; ++k, r += larger(step, r / 8 / step * step)) {
            if (total + (long long)units * (r - 1) > kMostTiles) return 0; // as much may the units count for
            if (padded(r) <= (long long)r * workers) return r;
        }
        return 0;
    };
    const int waves = workgroups * kPlanWaves, even = larger(kSoloTiles, quotient(total + waves - 1, waves));
    // an equal range wherever it begins: some wave has a unit's beginning more than the average
    const int anywhere = even + kPart + quotient(kPart * units, waves);
    int alone = fit(waves, 1);
    if (alone > anywhere) alone = 0;
    const int best = alone > 0 ? alone : anywhere, together = even <= kJoinBelow ? fit(workgroups, kPlanWaves) : 0;
    if (together > 0 && together <= kPlanWaves * (best + kJoin)) {
        per = round = together;
        return false;
    }
    per = alone > 0 ? larger(alone, kSoloTiles) : even;
    round = alone > 0 ? per : 1;
    return true;
}

} // namespace q4kv
