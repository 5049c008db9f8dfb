// A workgroup's wavefronts joining rows (csrc/join.h) on the CPU, one at a time and each as
// far ahead of the others as barriers let it: what one still has to read, another must not
// have written over.  A thread stands for a wavefront's first lane.
//
//   join_waves            rows with and without data in many orders; exit code 0: all right
//   join_waves by_rows    the halves given by the row's number instead of the joins': finds it wrong
#include <condition_variable>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <mutex>
#include <thread>
#include <vector>

#define __device__
static thread_local struct {
    int x;
} threadIdx;

struct Team {
    std::mutex mutex;
    std::condition_variable turn;
    std::vector<int> state;   // 0: may run, 1: at a barrier, 2: done
    int running = -1, first = 0;

    // under the lock: who runs next; all at the barrier are let go where nobody else may run
    void pass() {
        for (int again = 0; again < 2; again++) {
            const int n = (int)state.size();
            for (int k = 0; k < n; k++)
                if (state[(first + k) % n] == 0) {
                    running = (first + k) % n;
                    turn.notify_all();
                    return;
                }
            for (int &s : state) s = s == 1 ? 0 : s;
            first = (first + 1) % n;   // another one leads
        }
        running = -1;
    }
    void begin(int wave) {
        std::unique_lock<std::mutex> lock(mutex);
        turn.wait(lock, [&] { return running == wave; });
    }
    void barrier(int wave) {
        std::unique_lock<std::mutex> lock(mutex);
        state[wave] = 1;
        pass();
        turn.wait(lock, [&] { return running == wave; });
    }
    void end(int wave) {
        std::unique_lock<std::mutex> lock(mutex);
        state[wave] = 2;
        pass();
    }
};

static Team *team;
static void __syncthreads() { team->barrier(threadIdx.x / 64); }

#include "../paper_2601_17091_amd/csrc/join.h"

template <int WAVES, bool TOP>
int wrong(const std::vector<bool> &live, bool by_rows) {
    Team all;
    all.state.assign(WAVES, 0);
    team = &all;
    static float shared[4 * WAVES];
    int bad[WAVES] = {};
    std::vector<std::thread> waves;
    for (int wave = 0; wave < WAVES; wave++)
        waves.emplace_back([&, wave] {
            threadIdx.x = 64 * wave;
            all.begin(wave);
            int turn = 0;
            for (int row = 0; row < (int)live.size(); row++) {
                if (!live[row]) continue;
                if (by_rows) turn = row & 1;
                float s = (float)(row + 1) * (wave + 1);
                uint32_t top = (uint32_t)((row + 1) * 100 + (wave * 7 + row) % WAVES);
                rocket::join_waves<WAVES, TOP>(s, top, shared, turn);
                bad[wave] += s != (float)(row + 1) * (WAVES * (WAVES + 1) / 2);
                if (TOP) bad[wave] += top != (uint32_t)((row + 1) * 100 + WAVES - 1);
            }
            all.end(wave);
        });
    {
        std::unique_lock<std::mutex> lock(all.mutex);
        all.pass();
    }
    for (std::thread &t : waves) t.join();
    int sum = 0;
    for (int b : bad) sum += b;
    return sum;
}

template <int WAVES>
int both(const std::vector<bool> &live, bool by_rows) {
    return wrong<WAVES, false>(live, by_rows) + wrong<WAVES, true>(live, by_rows);
}

int main(int argc, char **argv) {
    const bool by_rows = argc > 1 && !strcmp(argv[1], "by_rows");
    int bad = 0;
    for (int pattern = 0; pattern < 128; pattern++) {   // every order of seven rows with and without data
        std::vector<bool> live(7);
        for (int k = 0; k < 7; k++) live[k] = pattern >> k & 1;
        bad += both<2>(live, by_rows) + both<4>(live, by_rows);
        if (pattern % 16 == 5) bad += both<8>(live, by_rows) + both<16>(live, by_rows);
    }
    printf("%d wrong\n", bad);
    return bad != 0;
}
