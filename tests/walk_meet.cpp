// Host-side check of how the waves of a workgroup meet over tiles in LDS (hp_meet.hpp, the kernels' own arithmetic):
// built by tests/test_operators_meet.py with UBSan.
// usage: walk_meet <loads|flag> <mistake>
//   loads: every wave of workgroups of 128 to 1024 lanes asks for tiles three ahead, two matrices a tile and the rows'
//   numbers by wave 0, and waits as the kernel does; no load of the tile that is then read may still be under way, and
//   no fewer tiles than were asked for after it (so that asking ahead is not undone).  mistake: waits go by
//   0: the wave's own loads; 1: those of the waves that make most.
//   flag: threads in the place of waves read a flag, some of them late, and the first clears it as soon as it goes on; all
//   have to have read the same.  mistake: the flag is read 0: as the kernels do; 1: behind one barrier and before none.
#include <chrono>
#include <condition_variable>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <deque>
#include <mutex>
#include <thread>
#include <vector>

#include "hp_meet.hpp"

#define CHECK(c, ...) \
    do { if (!(c)) { std::printf(__VA_ARGS__); std::printf(": %s\n", #c); return 1; } } while (0)

static int check_loads(int mistake) {
    for (int threads = 128; threads <= 1024; threads *= 2)
        for (int pieces = 64; pieces <= 2048; pieces += 64)
            for (int wave = 0; wave < threads / 64; ++wave) {
                int own = 0;                                      // counted round by round
                for (int at = 64 * wave; at < pieces; at += threads) ++own;
                const int most = hp::loads_of_wave(pieces, threads, 0), least = hp::loads_of_wave(pieces, threads, threads / 64 - 1);
                CHECK(hp::loads_of_wave(pieces, threads, wave) == own && (own == most || own == least), "%d pieces, %d lanes, wave %d", pieces, threads, wave);
                const int extra = wave == 0, each = 2 * (mistake ? most : own) + extra, stages = 4;
                for (int tiles = 1; tiles <= 9; ++tiles) {
                    std::deque<int> queue;                        // the tiles that loads under way belong to
                    const auto ask = [&](int t) { queue.insert(queue.end(), (size_t)(2 * own + extra), t); };
                    for (int t = 0; t < stages - 1 && t < tiles; ++t) ask(t);
                    for (int t = 0; t < tiles; ++t) {
                        const int left = tiles - t < stages - 1 ? tiles - t : stages - 1, behind = left - 1;
                        while ((int)queue.size() > hp::under_way(each, behind)) queue.pop_front();
                        CHECK(queue.empty() || queue.front() > t, "%d pieces, %d lanes, wave %d: tile %d of %d is read before it is there", pieces, threads, wave, t, tiles);
                        CHECK((int)queue.size() == behind * (2 * own + extra), "%d pieces, %d lanes, wave %d: tile %d of %d", pieces, threads, wave, t, tiles);
                        if (t + stages - 1 < tiles) ask(t + stages - 1);
                    }
                }
            }
    return 0;
}

class Barrier {
    std::mutex m;
    std::condition_variable all;
    int waiting = 0, turn = 0;
    const int n;

  public:
    explicit Barrier(int count) : n(count) {}
    void meet() {
        std::unique_lock<std::mutex> lock(m);
        const int mine = turn;
        if (++waiting == n) {
            waiting = 0, ++turn;
            all.notify_all();
        } else {
            all.wait(lock, [&] { return turn != mine; });
        }
    }
};

static int check_flag(int mistake) {
    for (int late = 0; late < 4; ++late) {                        // the wave that is held up behind every barrier
        constexpr int kWaves = 4;
        Barrier barrier(kWaves);
        int flag = 1, got[kWaves] = {};
        std::vector<std::thread> waves;
        for (int w = 0; w < kWaves; ++w)
            waves.emplace_back([&, w] {
                const auto meet = [&] {
                    barrier.meet();
                    if (w == late) std::this_thread::sleep_for(std::chrono::milliseconds(100));
                };
                if (mistake) {
                    meet();
                    got[w] = __atomic_load_n(&flag, __ATOMIC_RELAXED);
                } else {
                    got[w] = hp::read_together(&flag, meet);
                }
                if (w == 0) __atomic_store_n(&flag, 0, __ATOMIC_RELAXED);
            });
        for (std::thread &t : waves) t.join();
        for (int w = 0; w < kWaves; ++w) CHECK(got[w] == 1, "wave %d, with wave %d late, read another flag than wave 0", w, late);
    }
    return 0;
}

int main(int argc, char **argv) {
    if (argc != 3) return 2;
    int rc = 2;
    if (!std::strcmp(argv[1], "loads")) rc = check_loads(std::atoi(argv[2]));
    if (!std::strcmp(argv[1], "flag")) rc = check_flag(std::atoi(argv[2]));
    if (rc == 0) std::printf("ok\n");
    return rc;
}
