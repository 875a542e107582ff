// CPU stand-in for launches of any size: none but the workgroups that a test names are run, so that calls whose grids and buffers
// are far too large for a CPU can be looked at (buffers: address space of which few pages are touched).  Test infrastructure.
#pragma once
#include <hip/hip_runtime.h>

namespace some_workgroups {

struct Launch {
    uint64_t first;   // workgroups of the call before its own
    uint32_t groups, threads;
};
inline std::vector<Launch> launches;
inline std::vector<uint64_t> wanted;  // counted over all launches of a call
inline uint64_t seen = 0;

inline void run(uint32_t group, dim3 grid, dim3 block, const std::function<void()> &fn)
{
    hip_emul::BlockCtx ctx(block.x);
    std::vector<std::thread> lanes;
    for (unsigned t = 0; t < block.x; t++)
        lanes.emplace_back([&, t]() {
            hip_emul::ThreadState &s = hip_emul::tls;
            s.tid = dim3(t);
            s.bid = dim3(group);
            s.bdim = block;
            s.gdim = grid;
            s.ctx = &ctx;
            s.or_calls = 0;
            s.settled = false;
            fn();
            s.settle();
            ctx.ended++;
            ctx.wave_bar[t >> 6]->arrive_and_drop();
            ctx.bar.arrive_and_drop();
        });
    for (auto &l : lanes) l.join();
}

inline void launch(dim3 grid, dim3 block, const std::function<void()> &fn)
{
    launches.push_back({seen, grid.x, block.x});
    for (uint64_t w : wanted)
        if (w >= seen && w < seen + grid.x) run((uint32_t)(w - seen), grid, block, fn);
    seen += grid.x;
}

}  // namespace some_workgroups

#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, shmem, stream, ...) some_workgroups::launch((grid), (block), [&]() { kernel(__VA_ARGS__); })

extern "C" {
// names the workgroups to run from now on, and forgets the launches so far
inline __attribute__((used)) void some_workgroups_want(const uint64_t *groups, int n)
{
    some_workgroups::wanted.assign(groups, groups + n);
    some_workgroups::launches.clear();
    some_workgroups::seen = 0;
}
// launch i since then: {workgroups before it, workgroups, threads}; the number of launches
inline __attribute__((used)) int some_workgroups_launch(int i, uint64_t out[3])
{
    const int n = (int)some_workgroups::launches.size();
    if (i < n) {
        out[0] = some_workgroups::launches[i].first;
        out[1] = some_workgroups::launches[i].groups;
        out[2] = some_workgroups::launches[i].threads;
    }
    return n;
}
}
