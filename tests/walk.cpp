// The stages that the workgroups of a product of 8-bit rows ask for (csrc/walk.h), on the
// CPU: every stage of every tile once, and none whose columns begin past its buffers.
//
//   walk           exit code 0: all right
//   walk as_if     stages past the last tile begin where a tile's would: finds it wrong
#include <algorithm>
#include <cstdio>
#include <cstring>
#include <map>
#include <tuple>

#define __device__
#include "../paper_2601_17091_amd/csrc/walk.h"

struct Call {
    int64_t rows;
    int channels, columns, most_groups;
    int kM, kT, cols, slots, parts;
};

long wrong(const Call &c, bool as_if) {
    long bad = 0;
    const int tiles = (c.channels + c.kM - 1) / c.kM, all_stages = (c.columns + c.cols - 1) / c.cols;
    const int64_t tiles_t = (c.rows + c.kT - 1) / c.kT, items = tiles_t * tiles;
    const int each = (all_stages + c.parts - 1) / c.parts;
    const int64_t groups = c.parts > 1 ? items * c.parts : std::min<int64_t>(items, c.most_groups);
    std::map<std::tuple<int64_t, int, int>, int> seen;
    for (int64_t group = 0; group < groups; group++) {
        const int part = c.parts > 1 ? (int)(group % c.parts) : 0, stage0 = part * each;
        const int stages = c.parts > 1 ? std::min(all_stages - stage0, each) : all_stages;
        const int64_t first = c.parts > 1 ? group / c.parts : group;
        const rocket::Steps steps = {c.parts > 1 ? INT32_MAX : groups / tiles, (int)(groups % tiles), tiles};
        rocket::Tile tile = {first / tiles, (int)(first % tiles)};
        rocket::Asked asked = {tile, 0, true};
        int64_t weights = 0, rows = 0;
        const auto open_tile = [&]() {
            const int64_t first_t = asked.tile.t * c.kT, first_m = (int64_t)asked.tile.m * c.kM;
            asked.there = first_t < c.rows;
            weights = asked.there ? rocket::bytes_of_lines(c.channels, first_m, c.kM, c.columns) : 0;
            rows = rocket::bytes_of_lines(c.rows, first_t, c.kT, c.columns);
            bad += asked.tile.m < 0 || asked.tile.m >= tiles || asked.there != (rows > 0);
        };
        const auto ask = [&]() {
            if (asked.crosses(stages, steps)) open_tile();
            const int stage = stage0 + asked.stage;
            if (as_if) asked.there = true;
            const int64_t at = asked.next(stage0, c.cols);
            if (rows > 0) seen[{asked.tile.t, asked.tile.m, stage}]++;
            if (rows > 0) bad += at != (int64_t)stage * c.cols || at >= c.columns;
            bad += at > weights || at > rows;
        };
        open_tile();
        for (int k = 0; k < c.slots; k++) ask();
        for (; tile.t < tiles_t; tile = steps.after(tile))
            for (int stage = 0; stage < stages; stage++) ask();
    }
    for (const auto &s : seen) bad += s.second != 1;
    return bad + ((int64_t)seen.size() != items * all_stages);
}

int main(int argc, char **argv) {
    const bool as_if = argc > 1 && !strcmp(argv[1], "as_if");
    long bad = 0;
    const int ways[][4] = {{256, 256, 128, 2}, {256, 128, 128, 2}, {128, 128, 128, 3}, {128, 128, 64, 3}, {64, 64, 64, 4}};
    for (const auto &w : ways)
        for (int64_t rows : {65, 128, 129, 1000, 5001})
            for (int channels : {1, 64, 257, 993, 2000})
                for (int columns : {64, 128, 192, 960, 2048})
                    for (int groups : {7, 256, 512})
                        bad += wrong({rows, channels, columns, groups, w[0], w[1], w[2], w[3], 1}, as_if);
    for (int64_t rows : {65, 300, 1000})
        for (int channels : {33, 190, 2000})
            for (int columns : {4096, 8192, 20032})
                for (int parts : {2, 5, 16})
                    bad += wrong({rows, channels, columns, 256, 128, 128, 128, 3, parts}, as_if);
    printf("%ld wrong\n", bad);
    return bad != 0;
}
