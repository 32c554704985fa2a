// Which sequence a slot of the ragged attention belongs to: the arithmetic of the search, for any 64 lanes (a wavefront's in
// avion_ragged.h, an array's on the host, where it can be tested for every number of sequences).
//
// The borders of the S + 2 intervals (rows before the first sequence, the sequences, rows behind the last one) are 0, the offsets and T;
// interval i begins at slot floor(border_i mul / 2^SHIFT) + i, so that those places grow strictly.  A step probes 63 of the intervals that are
// left, evenly spread, one a lane, and goes on among those from the last one that has begun to the next probe: 61 sequences take one step,
// 3967 two, 250045 three and 2^20 four.
#pragma once

struct RaggedPlace {
    int i;         // interval of the borders (0 and S + 1: rows of no sequence)
    int begin, n;  // its tokens
    long block;    // of BM rows
};

// border i of 0 .. S + 2, held inside the tensor
__attribute__((always_inline)) constexpr int ragged_border(const int* off, int S, int T, int i)
{
    if (i <= 0) return 0;
    if (i > S + 1) return T;
    const int at = off[i - 1] > 0 ? off[i - 1] : 0;
    return at < T ? at : T;
}

// Lanes: load(lo, step) gives lane l border lo + l * step; count(f): how many of the 64 lanes have f(l, their border); at(l): lane l's border.
// The last step is always one of width 1: only then does the lane behind the one that is found hold the end of its interval.  (A wider
// step may leave a single interval too, whose end no lane holds: of 4031 sequences, probed 65 apart, every 65th.)
template <int SHIFT, typename Lanes>
__attribute__((always_inline)) constexpr RaggedPlace ragged_search(Lanes& lanes, int S, int mul, long slot)
{
    int lo = 0, n = S + 2, step = 0, c = 0;
    do {
        step = (n + 62) / 63;
        lanes.load(lo, step);
        const int begun = lanes.count([=](int lane, int border) {
            const int at = lane * step;
            return at < n && (((long)border * mul) >> SHIFT) + lo + at <= slot;
        });
        c = begun > 1 ? begun - 1 : 0;
        lo += c * step;
        n = step < n - c * step ? step : n - c * step;
    } while (step > 1);
    const int begin = lanes.at(c), end = lanes.at(c + 1);
    return RaggedPlace{lo, begin, end > begin ? end - begin : 0, slot - (((long)begin * mul) >> SHIFT) - lo};
}
