// The order that csrc/grkan_turns.h gives eight wavefronts, looked over on the host: what each of them does between which barriers is
// written down, and then every read from LDS is held against the loads of all.
#include <cstdint>
#include <cstdio>
#include <vector>

#define __device__
#define __forceinline__ inline
#include "../../paper_2505_13813_amd/csrc/grkan_turns.h"

constexpr uint32_t kPlace = 16384;
constexpr int kWaves = 8, kNever = 1 << 30;

enum Kind { KEYS, VALUES };
struct Event {
    Kind kind;
    int32_t pass, tile;
    uint32_t place;
    int turn;   // barriers in front of it
    int landed; // of a load: barriers in front of the wait that it is known to have landed by
};
struct Wave {
    std::vector<Event> loads, reads;
    int turn = 0;
};

// Two passes, as where the first one's sums are not finite.
static Wave run(int32_t tiles, bool second)
{
    Wave w;
    for (int32_t pass = 0; pass < 2; ++pass) {
        auto wait = [&] {
            for (Event &e : w.loads)
                if (e.landed == kNever)
                    e.landed = w.turn;
        };
        auto meet = [&] { ++w.turn; };
        auto load = [&](Kind kind, int32_t t, uint32_t at) {
            if (t < tiles)
                w.loads.push_back(Event{kind, pass, t, at, w.turn, kNever});
        };
        auto read = [&](Kind kind, int32_t t, uint32_t at) {
            if (t < tiles)
                w.reads.push_back(Event{kind, pass, t, at, w.turn, 0});
        };
        if (pass > 0) {
            wait();
            meet();
        }
        load(KEYS, 0, 0);
        grkan::attention::take_turns<kPlace>(
            tiles, second, wait, meet, [&](int32_t t, uint32_t at) { load(KEYS, t, at); }, [&](int32_t t, uint32_t at) { load(VALUES, t, at); },
            [&] { read(KEYS, 0, 0); }, [](int32_t, uint32_t, uint32_t) {},
            [&](int32_t t, uint32_t at, uint32_t next, uint32_t last) {
                load(KEYS, t + 3, at);
                load(VALUES, t + 2, last);
                read(KEYS, t + 1, next);
                read(VALUES, t, at);
            });
    }
    return w;
}

static int faults_of(int32_t tiles)
{
    std::vector<Wave> waves;
    for (int w = 0; w < kWaves; ++w)
        waves.push_back(run(tiles, w >= 4));
    int faults = 0;
    auto fault = [&](const char *what, int w, const Event &e, int by) {
        std::printf("%d tiles: wavefront %d, pass %d, %s of tile %d behind barrier %d: %s %d\n", tiles, w, e.pass, e.kind == KEYS ? "keys" : "values", e.tile, e.turn,
                    what, by);
        ++faults;
    };
    for (int w = 0; w < kWaves; ++w) {
        if (waves[w].turn != waves[0].turn) {
            std::printf("%d tiles: wavefront %d meets %d times, the first %d times\n", tiles, w, waves[w].turn, waves[0].turn);
            ++faults;
        }
        if (waves[w].reads.size() != 2u * 2u * (unsigned)tiles) {
            std::printf("%d tiles: wavefront %d reads %zu times\n", tiles, w, waves[w].reads.size());
            ++faults;
        }
        for (const Event &r : waves[w].reads)
            for (int o = 0; o < kWaves; ++o) {
                int there = 0;
                for (const Event &l : waves[o].loads) {
                    if (l.kind != r.kind || l.place != r.place)
                        continue;
                    if (l.pass == r.pass && l.tile == r.tile) {
                        ++there;
                        if (l.landed >= r.turn)
                            fault("not waited for in front of it by wavefront", w, r, o);
                    } else if (l.pass > r.pass || (l.pass == r.pass && l.tile > r.tile)) {
                        if (l.turn <= r.turn)
                            fault("its place may be loaded to already by wavefront", w, r, o);
                    } else if (l.landed >= r.turn) {
                        fault("what was there before may still come in, of wavefront", w, r, o);
                    }
                }
                if (there != 1)
                    fault("loads of its part by wavefront", w, r, o);
            }
    }
    return faults;
}

int main()
{
    int faults = 0;
    for (int32_t tiles = 1; tiles < 12; ++tiles)
        faults += faults_of(tiles);
    if (faults == 0)
        std::printf("in order\n");
    return faults != 0;
}
