// Host model of the ring between the TMA warp, the converter warps and the MMA warp of the score-cache kernel, around the turns
// that the kernel itself is compiled from (converter_turns.cuh).  Barriers behave like mbarriers whose waits look at a parity; the
// warps run in random order, some of them much slower than others for a while.
// Arguments: raw stages, operand slots, tiles per unit, units, seeds.  Prints the runs that got stuck or met a wrong tile.
#include <ucontext.h>

#include <cstdio>
#include <cstdlib>
#include <functional>
#include <memory>
#include <random>
#include <vector>

#include "converter_turns.cuh"

namespace {

struct Bar {
    int count, pending;
    uint32_t phase = 0;
    explicit Bar(int n) : count(n), pending(n) {}
    void arrive()
    {
        if (--pending == 0) {
            pending = count;
            ++phase;
        }
    }
    bool passed(uint32_t parity) const { return (phase & 1) != (parity & 1); }
};

struct Warp {
    ucontext_t ctx;
    std::vector<char> stack;
    std::function<void()> body;
    bool done = false;
};

std::vector<std::unique_ptr<Warp>> warps;
ucontext_t scheduler;
int running;
long progress;  // waits that were passed
bool wrong;

void yield() { swapcontext(&warps[running]->ctx, &scheduler); }
void wait(const Bar& b, uint32_t parity)
{
    do yield();  // before the first look: a warp may be late at any of them
    while (!b.passed(parity));
    ++progress;
}
void start()
{
    warps[running]->body();
    warps[running]->done = true;
    yield();
}
void spawn(std::function<void()> body)
{
    warps.emplace_back(new Warp);
    Warp& w = *warps.back();
    w.body = std::move(body);
    w.stack.resize(64 * 1024);
    getcontext(&w.ctx);
    w.ctx.uc_stack.ss_sp = w.stack.data();
    w.ctx.uc_stack.ss_size = w.stack.size();
    w.ctx.uc_link = nullptr;
    makecontext(&w.ctx, start, 0);
}
void resume(int i)
{
    running = i;
    if (!warps[i]->done) swapcontext(&scheduler, &warps[i]->ctx);
}

// 0: every tile came through; 1: no warp can go on; 2: a tile was read before it was there or written before it was used
int run(int n_raw, int n_slots, int n_tiles, int units, unsigned seed)
{
    std::mt19937 rng(seed);
    std::vector<Bar> raw_full(n_raw, Bar(1)), raw_empty(n_raw, Bar(spec::kConverterArrivals)),
        slot_full(n_slots, Bar(spec::kConverterArrivals)), slot_empty(n_slots, Bar(1));
    struct Place { int tile = -1, parts = 2; };  // a tile's number, and the warps that have expanded their part of it
    std::vector<Place> raw(n_raw), slot(n_slots);
    const int all = n_tiles * units;
    warps.clear();
    progress = 0;
    wrong = false;
    spawn([&] {  // TMA
        for (int g = 0; g < all; ++g) {
            const int r = g % n_raw;
            wait(raw_empty[r], (g / n_raw & 1) ^ 1);
            wrong |= raw[r].parts != 2;
            raw[r].tile = g;
            raw[r].parts = 0;
            yield();  // the copy takes its time
            raw_full[r].arrive();
        }
    });
    for (int w = 0; w < spec::kConverterWarps; ++w)
        spawn([&, w] {
            spec::ConverterTurns t;
            for (int u = 0; u < units; ++u)
                spec::converter_tiles(
                    t, n_tiles, w / 2, n_raw, n_slots,
                    [&](uint32_t r, uint32_t rph, uint32_t sl, uint32_t sph) {
                        wait(raw_full[r], rph);
                        wait(slot_empty[sl], sph);
                        return true;
                    },
                    [&](uint32_t r, uint32_t sl) {
                        wrong |= raw[r].tile != (int)t.g || raw[r].parts >= 2;
                        yield();
                        ++raw[r].parts;
                        if (slot[sl].tile != (int)t.g) {
                            slot[sl].tile = (int)t.g;
                            slot[sl].parts = 0;
                        }
                        ++slot[sl].parts;
                    },
                    [&](uint32_t r, uint32_t sl) {
                        slot_full[sl].arrive();
                        raw_empty[r].arrive();
                    });
        });
    spawn([&] {  // MMA
        for (int g = 0; g < all; ++g) {
            const int s = g % n_slots;
            wait(slot_full[s], g / n_slots & 1);
            wrong |= slot[s].tile != g || slot[s].parts != 2;
            slot_empty[s].arrive();
        }
    });
    const int n = (int)warps.size();
    for (;;) {
        std::vector<double> speed(n);
        for (double& s : speed) s = rng() % 3 ? 1.0 : 0.002;
        std::discrete_distribution<int> pick(speed.begin(), speed.end());
        for (int i = 0; i < 200; ++i) resume(pick(rng));
        if (wrong) return 2;
        const long before = progress;  // in the end everybody gets a few turns
        bool over = true;
        for (int i = 0; i < 8 * n; ++i) resume(i % n);
        for (const auto& w : warps) over &= w->done;
        if (wrong) return 2;
        if (over) return 0;
        if (progress == before) return 1;
    }
}

}  // namespace

int main(int argc, char** argv)
{
    if (argc != 6) return 2;
    const int n_raw = atoi(argv[1]), n_slots = atoi(argv[2]), n_tiles = atoi(argv[3]), units = atoi(argv[4]), seeds = atoi(argv[5]);
    int stuck = 0, bad = 0;
    for (int s = 0; s < seeds; ++s) {
        const int r = run(n_raw, n_slots, n_tiles, units, 1000 * n_raw + 100 * n_slots + s);
        stuck += r == 1;
        bad += r == 2;
    }
    printf("%d %d\n", stuck, bad);
    return 0;
}
