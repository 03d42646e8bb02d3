// The search for a workgroup's tile in packed sequences (csrc/grkan_packed.h), run on the host as a wavefront runs it: 64 lanes, each a
// context of its own, that meet at every operation across lanes.
//
// Rising offsets: every tile of every segment once, the longest walks of 64 segments first.  Falling ones: whatever comes out lies in the
// buffer, and its place among the places.
#include <ucontext.h>

#include <algorithm>
#include <array>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <set>
#include <type_traits>
#include <utility>
#include <vector>

#define __device__
#define __forceinline__ inline

// ---- 64 lanes

struct Lane {
    ucontext_t context;
    std::vector<char> stack = std::vector<char>(64 * 1024);
    int operation;
    int64_t given;
    bool done;
};
static Lane lanes[64];
static int64_t settled[64];
static ucontext_t scheduler;
static int current;
static void (*program)(int);

enum { BALLOT = 1, READ, FIRST, SWAP16, SWAP32, DPP };

// what every lane gives at the same operation
static const int64_t *meet(int operation, int64_t given)
{
    lanes[current].operation = operation;
    lanes[current].given = given;
    swapcontext(&lanes[current].context, &scheduler);
    return settled;
}
static void start()
{
    program(current);
    lanes[current].done = true;
    swapcontext(&lanes[current].context, &scheduler);
}
static void run(void (*of_lane)(int))
{
    program = of_lane;
    for (Lane &l : lanes) {
        l.done = false;
        getcontext(&l.context);
        l.context.uc_stack.ss_sp = l.stack.data();
        l.context.uc_stack.ss_size = l.stack.size();
        l.context.uc_link = nullptr;
        makecontext(&l.context, start, 0);
    }
    for (;;) {
        int done = 0;
        for (current = 0; current < 64; ++current) {
            swapcontext(&scheduler, &lanes[current].context);
            done += lanes[current].done;
        }
        if (done == 64)
            return;
        for (const Lane &l : lanes)
            if (done || l.operation != lanes[0].operation) {
                std::printf("the lanes part\n");
                std::exit(1);
            }
        for (int i = 0; i < 64; ++i)
            settled[i] = lanes[i].given;
    }
}

static struct {
    struct {
        operator uint32_t() const { return (uint32_t)current; }
    } x;
} threadIdx;

static uint64_t __ballot(bool v)
{
    const int64_t *const all = meet(BALLOT, v);
    uint64_t bits = 0;
    for (int i = 0; i < 64; ++i)
        bits |= (uint64_t)(all[i] != 0) << i;
    return bits;
}
static int __popcll(uint64_t v) { return __builtin_popcountll(v); }
static int32_t __builtin_amdgcn_readlane(int32_t v, int32_t lane) { return (int32_t)meet(READ, v)[lane & 63]; }
static int32_t __builtin_amdgcn_readfirstlane(int32_t v) { return (int32_t)meet(FIRST, v)[0]; }
static int32_t __builtin_amdgcn_update_dpp(int32_t, int32_t v, int control, int, int, bool)
{
    const int64_t *const all = meet(DPP + control, v);
    const int i = current, quad = i & ~3;
    if (control < 0x100) // a quad's lanes, two bits for each
        return (int32_t)all[quad + (control >> 2 * (i & 3) & 3)];
    return (int32_t)all[control == 0x141 ? (i & ~7) + 7 - (i & 7) : (i & ~15) + 15 - (i & 15)]; // eight or sixteen mirrored
}
// odd rows of 16 (the upper 32) of the first operand for even rows (the lower 32) of the second
static std::array<uint32_t, 2> swapped(int operation, int by, uint32_t v)
{
    const int64_t *const all = meet(operation, v);
    const int i = current;
    return {(uint32_t)all[i & ~by], (uint32_t)all[i | by]};
}
static std::array<uint32_t, 2> __builtin_amdgcn_permlane16_swap(uint32_t v, uint32_t, bool, bool) { return swapped(SWAP16, 16, v); }
static std::array<uint32_t, 2> __builtin_amdgcn_permlane32_swap(uint32_t v, uint32_t, bool, bool) { return swapped(SWAP32, 32, v); }

// ---- what the header takes from others and the search has no part in

#define GRKAN_ATTENTION_H_
typedef int grkan_status_t, grkan_dtype_t;
struct grkan_causal_attention_t;
namespace grkan {
namespace attention {
struct u32x4 {
};
struct Operand {
    uint64_t at;
    int64_t batch, token, head;
};
struct Args {
    int64_t rows;
    int32_t kv_heads, group, dim;
};
template <int DP> constexpr uint32_t kBlock = 1024u;
template <int DP> constexpr uint32_t swizzle(uint32_t) { return 0; }
inline void lds_write16(uint32_t, u32x4) {}
inline void load_to_lds(uint64_t, uint32_t, uint32_t) {}
inline uint64_t uniform_u64(uint64_t v) { return v; }
inline uint32_t lane_here() { return 0; }
inline int64_t row_offset(uint32_t row, uint32_t group, int64_t token, int64_t head) { return (int64_t)(row / group) * token + (int64_t)(row % group) * head; }
} // namespace attention
} // namespace grkan

#include "../../paper_2505_13813_amd/csrc/grkan_packed.h"

using namespace grkan::attention;

// ---- the cases

static Packed operand;
static int32_t slot, unit;
static bool forward;
static Segment found[64];
template <int SIZE> static void search(int lane) { found[lane] = segment_of<SIZE>(operand, slot, unit, forward); }

static int faults = 0;
static void fault(const char *what, int size)
{
    std::printf("tiles of %d, unit %d, %d sequences, slot %d: %s\n", size, unit, operand.sequences, slot, what);
    ++faults;
}

template <int SIZE> static void check(const std::vector<int64_t> &ends, bool rising)
{
    const int32_t segments = operand.sequences + 2;
    const int64_t places = slots_of<SIZE>(operand, unit);
    std::set<std::pair<int32_t, int32_t>> seen;
    int64_t last = -1;
    int32_t of = -1; // the 64 segments
    for (slot = 0; slot < places; ++slot) {
        run(search<SIZE>);
        const Segment &s = found[0];
        for (const Segment &o : found)
            if (o.first != s.first || o.count != s.count || o.tile != s.tile || o.index != s.index || o.none != s.none)
                fault("lanes do not agree", SIZE);
        const bool there = (int64_t)s.tile * SIZE < (int64_t)s.count * unit;
        if (s.first < 0 || s.count < 0 || (int64_t)s.first + s.count > operand.tokens || s.tile < 0 || s.index < 0 || s.index >= segments)
            fault("out of the buffer", SIZE);
        if (s.none != (s.index == 0 || s.index == segments - 1))
            fault("whether it is a sequence", SIZE);
        if (s.count == 0 && s.tile != 0)
            fault("a tile of nothing", SIZE);
        if (!there)
            continue;
        if (place_of<SIZE>(s.first, unit, s.index) + s.tile >= places)
            fault("no place for it", SIZE);
        if (rising) {
            if (s.first != ends[s.index] || s.first + s.count != ends[s.index + 1])
                fault("another segment", SIZE);
            if (!seen.insert({s.index, s.tile}).second)
                fault("twice", SIZE);
            const int64_t tiles = ((int64_t)s.count * unit + SIZE - 1) / SIZE, walk = forward ? s.tile : tiles - 1 - s.tile;
            if (s.index / 64 == of && walk > last)
                fault("a longer walk behind a shorter one", SIZE);
            of = s.index / 64;
            last = walk;
        }
    }
    slot = -1;
    if (rising)
        for (int32_t i = 0; i < segments; ++i)
            for (int64_t t = 0; t * SIZE < (ends[i + 1] - ends[i]) * unit; ++t)
                if (!seen.count({i, (int32_t)t}))
                    fault("a tile is nobody's", SIZE);
}

int main()
{
    std::mt19937 random(1);
    auto upto = [&](int64_t n) { return (int64_t)(random() % (uint64_t)(n + 1)); };
    const int counts[] = {0, 1, 2, 5, 30, 61, 62, 63, 64, 126, 127, 200};
    int ran = 0;
    for (int round = 0; round < 36; ++round) {
        const int sequences = counts[round % 12], kind = round % 5; // kind 3: of one length, without offsets; 4: falling ones among them
        const int64_t front = kind == 3 ? 0 : upto(2) * upto(70), behind = kind == 3 ? 0 : upto(2) * upto(70), each = upto(40);
        std::vector<int64_t> offsets{front};
        for (int i = 0; i < sequences; ++i) {
            const int64_t lengths[] = {0, 1, upto(30), upto(sequences > 30 ? 40 : 500)};
            offsets.push_back(offsets.back() + (kind == 3 ? each : lengths[upto(3)]));
        }
        const int64_t tokens = kind == 3 && sequences == 0 ? 0 : offsets.back() + behind;
        std::vector<int64_t> ends{0};
        ends.insert(ends.end(), offsets.begin(), offsets.end());
        ends.push_back(tokens);
        const bool rising = kind != 4;
        if (!rising)
            for (int64_t &o : offsets)
                o = upto(tokens + 100) - 50;
        std::vector<int32_t> narrow(offsets.begin(), offsets.end());
        operand = Packed{};
        operand.tokens = (int32_t)tokens;
        operand.sequences = sequences;
        operand.offsets_64 = round % 2;
        operand.offsets = kind == 3 ? nullptr : operand.offsets_64 ? (const void *)offsets.data() : (const void *)narrow.data();
        operand.each = (int32_t)each;
        const int units[] = {1, 1, 2, 3, 7, 40};
        unit = units[upto(tokens > 2000 ? 2 : 5)];
        forward = round / 2 % 2;
        switch (round % 4) {
        case 0:
            check<32>(ends, rising);
            break;
        case 1:
            check<64>(ends, rising);
            break;
        case 2:
            check<128>(ends, rising);
            break;
        default:
            check<256>(ends, rising);
        }
        ++ran;
    }
    // a sequence behind others that fall again and again: more tiles than places
    std::vector<int64_t> saw{0};
    for (int i = 0; i < 6; ++i)
        saw.insert(saw.end(), {1000, 0});
    saw.insert(saw.end(), {1000, 1100});
    operand = Packed{};
    operand.tokens = 1100;
    operand.sequences = (int32_t)saw.size() - 1;
    operand.offsets = saw.data();
    operand.offsets_64 = 1;
    for (int i = 0; i < 4; ++i) {
        unit = 1 + 3 * (i / 2);
        forward = i % 2;
        check<64>(saw, false);
    }
    if (faults == 0 && ran == 36)
        std::printf("every tile once\n");
    return faults != 0;
}
