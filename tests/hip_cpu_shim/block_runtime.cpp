// Runtime behind block_lanes.hpp: workgroups one after the other, their lanes as fibres (test infrastructure only).
#include "block_lanes.hpp"

#include <sanitizer/common_interface_defs.h>
#include <sys/mman.h>
#include <ucontext.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <deque>

thread_local shim_uint3 threadIdx, blockIdx;
thread_local dim3 blockDim, gridDim;

// compiler-rt's conversion, which the compiler calls for (__bf16)x on the host: to nearest even
extern "C" __bf16 __truncsfbf2(float x)
{
    uint32_t u = __float_as_uint(x);
    if (x != x) u |= 0x400000u;
    else u += 0x7FFFu + (u >> 16 & 1u);
    const uint16_t half = (uint16_t)(u >> 16);
    __bf16 out;
    std::memcpy(&out, &half, 2);
    return out;
}

namespace shim {
thread_local unsigned char *dyn_smem = nullptr;
thread_local unsigned char *lds = nullptr;
int compute_units = 8, blocks_per_cu = 4, force = -1;
size_t max_dynamic_lds = 160 * 1024;
std::atomic<long> launches{0}, streaming_loads{0}, largest_launch{0};
bool dry_run = false;

namespace {
constexpr int kWave = 64;
constexpr size_t kStack = 256 * 1024;
enum class At { ready, wave, block, done };
struct Copy {
    unsigned char *to;
    const void *from;
};
struct Lane {
    ucontext_t ctx;
    char *stack = nullptr;
    void *fake = nullptr;
    At at = At::done;
    size_t shared = 0;                                // __shared__ arrays that it has come to
    std::deque<Copy> copies;
    alignas(16) unsigned char slots[2][64];           // what it exchanges, in turns: who writes one again has met the others since they read it
    int turn = 0;
};
std::vector<Lane> lanes;
std::vector<void *> arrays;
int count = 0, running = 0, last_error = hipSuccess;
ucontext_t scheduler;
void *scheduler_fake = nullptr;
const void *scheduler_bottom = nullptr;
size_t scheduler_size = 0;
const std::function<void()> *body = nullptr;

void leave(At at)
{
    Lane &me = lanes[running];
    me.at = at;
    __sanitizer_start_switch_fiber(at == At::done ? nullptr : &me.fake, scheduler_bottom, scheduler_size);
    swapcontext(&me.ctx, &scheduler);
    __sanitizer_finish_switch_fiber(me.fake, &scheduler_bottom, &scheduler_size);
}

void lane_main()
{
    __sanitizer_finish_switch_fiber(nullptr, &scheduler_bottom, &scheduler_size);
    (*body)();
    if (!lanes[running].copies.empty()) {
        std::fprintf(stderr, "shim: a lane ends with copies that it never waited for\n");
        std::abort();
    }
    leave(At::done);
}

// Lets every lane of [from, to) that is at `where` go on, if all that have not returned are there.
bool release(int from, int to, At where)
{
    bool any = false;
    for (int l = from; l < to; l++) {
        if (lanes[l].at == where) any = true;
        else if (lanes[l].at != At::done) return false;
    }
    if (any)
        for (int l = from; l < to; l++)
            if (lanes[l].at == where) lanes[l].at = At::ready;
    return any;
}

void run_workgroup()
{
    arrays.clear();
    for (int l = 0; l < count; l++) {
        Lane &lane = lanes[l];
        getcontext(&lane.ctx);
        lane.ctx.uc_stack = {lane.stack, 0, kStack};
        lane.ctx.uc_link = nullptr;
        lane.at = At::ready;
        lane.shared = 0;
        lane.fake = nullptr;
        makecontext(&lane.ctx, lane_main, 0);
    }
    for (;;) {
        bool ran = false;
        for (int w = 0; w < count; w += kWave) {
            const int end = std::min(w + kWave, count);
            do {                                      // a wavefront as far as it comes by itself
                for (int l = w; l < end; l++)
                    if (lanes[l].at == At::ready) {
                        ran = true;
                        running = l;
                        threadIdx = {(unsigned)l, 0, 0};
                        __sanitizer_start_switch_fiber(&scheduler_fake, lanes[l].stack, kStack);
                        swapcontext(&scheduler, &lanes[l].ctx);
                        __sanitizer_finish_switch_fiber(scheduler_fake, nullptr, nullptr);
                    }
            } while (release(w, end, At::wave));
        }
        if (release(0, count, At::block)) continue;
        if (!ran) break;
    }
    for (int l = 0; l < count; l++)
        if (lanes[l].at != At::done) {
            std::fprintf(stderr, "shim: lane %d of workgroup %u waits for others that do not come\n", l, blockIdx.x);
            std::abort();
        }
    for (void *p : arrays) std::free(p);
}

// Hands `bytes` to the wavefront; returns when all its lanes have.
void give(const void *mine, size_t bytes)
{
    Lane &me = lanes[running];
    me.turn ^= 1;
    std::memcpy(me.slots[me.turn], mine, bytes);
    leave(At::wave);
}
const unsigned char *of_lane(int lane)                // of the wavefront, which may have gone on meanwhile
{
    const int l = running / kWave * kWave + lane;
    return lanes[l].slots[lanes[running].turn];
}

float number(uint16_t bits, bool bf)
{
    if (bf) return __uint_as_float((uint32_t)bits << 16);
    _Float16 h;
    std::memcpy(&h, &bits, 2);
    return (float)h;
}

// lane l has row l % SIZE of either side, eight k from 8 (l / SIZE) on; of the result column l % SIZE, rows in fours.  (The loop is
// most of what a run does, on numbers of its own: left to the compiler as it is.)
template <int SIZE, int K, int RESULTS>
__attribute__((no_sanitize("address", "undefined"))) void multiply_any(const uint16_t *a, const uint16_t *b, bool bf, float *c)
{
    float both[16];
    for (int i = 0; i < 8; i++) both[i] = number(a[i], bf), both[8 + i] = number(b[i], bf);
    give(both, sizeof both);
    const int lane = running % kWave, column = lane % SIZE, group = lane / SIZE;
    const int turn = lanes[running].turn;
    const Lane *const wave = lanes.data() + running / kWave * kWave;
    for (int i = 0; i < RESULTS; i++) {
        const int row = SIZE == 16 ? 4 * group + i : 8 * (i / 4) + 4 * group + i % 4;
        float sum = c[i];
        for (int k = 0; k < K; k += 8) {
            const float *left = reinterpret_cast<const float *>(wave[row + k / 8 * SIZE].slots[turn]);
            const float *right = reinterpret_cast<const float *>(wave[column + k / 8 * SIZE].slots[turn]) + 8;
            for (int e = 0; e < 8; e++) sum += left[e] * right[e];
        }
        c[i] = sum;
    }
}
}  // namespace

void barrier_wait() { leave(At::block); }

void *block_shared(size_t bytes, size_t align)
{
    Lane &me = lanes[running];
    if (me.shared == arrays.size()) {
        void *p = nullptr;
        if (posix_memalign(&p, align, bytes)) std::abort();
        std::memset(p, 0xFF, bytes);                  // NaN to whoever reads what nobody has written
        arrays.push_back(p);
    }
    return arrays[me.shared++];
}

void wave_in_step() { leave(At::wave); }

uint32_t read_lane(uint32_t v, int lane)
{
    give(&v, 4);
    std::memcpy(&v, of_lane(lane), 4);
    return v;
}

uint32_t update_dpp(uint32_t old, uint32_t v, int control, int rows, int banks, bool bound)
{
    if (banks != 15 || !bound) std::abort();
    give(&v, 4);
    const int lane = running % kWave;
    uint32_t got = 0;
    if (control > 0x110 && control < 0x120) {         // shifted up within sixteen lanes
        if (lane % 16 >= control - 0x110) std::memcpy(&got, of_lane(lane - (control - 0x110)), 4);
    } else if (control == 0x142) {                    // the last of each sixteen to the next
        if (lane >= 16) std::memcpy(&got, of_lane(lane / 16 * 16 - 1), 4);
    } else if (control == 0x143) {                    // lane 31 to the upper half
        if (lane >= 32) std::memcpy(&got, of_lane(31), 4);
    } else {
        std::abort();
    }
    return rows >> (lane / 16) & 1 ? got : old;
}

void copy_to_lds(uint32_t to, const void *from)
{
    lanes[running].copies.push_back({lds + to + running % kWave * 16, from});
}

__attribute__((optnone)) static void arrive(const Copy &c)       // byte by byte, each of them checked
{
    for (int i = 0; i < 16; i++) c.to[i] = static_cast<const unsigned char *>(c.from)[i];
}

void wait_copies(int but)
{
    auto &copies = lanes[running].copies;
    for (; (int)copies.size() > but; copies.pop_front()) arrive(copies.front());
}

Bits4 read_transposed(const void *lane_address)
{
    short four[4];
    std::memcpy(four, lane_address, 8);
    give(four, 8);
    const int lane = running % kWave, of = lane % 16;
    Bits4 out;
    for (int r = 0; r < 4; r++) {
        short v;
        std::memcpy(&v, of_lane(lane / 16 * 16 + r * 4 + of / 4) + of % 4 * 2, 2);
        out[r] = v;
    }
    return out;
}

void multiply16(const uint16_t *a, const uint16_t *b, bool bf, float *c) { multiply_any<16, 32, 4>(a, b, bf, c); }
void multiply32(const uint16_t *a, const uint16_t *b, bool bf, float *c) { multiply_any<32, 16, 16>(a, b, bf, c); }

void launch(dim3 grid, dim3 block, size_t bytes, const std::function<void()> &kernel)
{
    launches++;
    if (!grid.x || !grid.y || !grid.z || grid.y > 65535 || grid.z > 65535 || !block.x || block.x > 1024 || block.y != 1 || block.z != 1 || bytes ||
        (uint64_t)grid.x * block.x >> 32) {
        std::fprintf(stderr, "shim: launch refused (grid %u %u %u, block %u)\n", grid.x, grid.y, grid.z, block.x);
        last_error = hipErrorInvalidValue;
        return;
    }
    if (dry_run) return;
    blockDim = block;
    gridDim = grid;
    body = &kernel;
    count = (int)block.x;
    while (lanes.size() < (size_t)count) {
        lanes.emplace_back();
        lanes.back().stack = static_cast<char *>(mmap(nullptr, kStack, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0));
        if (lanes.back().stack == MAP_FAILED) std::abort();
    }
    for (unsigned z = 0; z < grid.z; z++)
        for (unsigned y = 0; y < grid.y; y++)
            for (unsigned x = 0; x < grid.x; x++) {
                blockIdx = {x, y, z};
                run_workgroup();
            }
}
}  // namespace shim

hipError_t hipMalloc(void **p, size_t bytes)
{
    *p = std::malloc(bytes ? bytes : 1);
    if (!*p) return hipErrorOutOfMemory;
    std::memset(*p, 0xFF, bytes);
    return hipSuccess;
}
hipError_t hipFree(void *p) { std::free(p); return hipSuccess; }
hipError_t hipMemcpy(void *dst, const void *src, size_t bytes, hipMemcpyKind) { std::memcpy(dst, src, bytes); return hipSuccess; }
hipError_t hipGetDevice(int *dev) { *dev = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipGetLastError() { const int e = shim::last_error; shim::last_error = hipSuccess; return e; }
hipError_t hipDeviceGetAttribute(int *out, hipDeviceAttribute_t, int) { *out = shim::compute_units; return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t *ev, unsigned) { *ev = reinterpret_cast<hipEvent_t>(std::malloc(1)); return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t ev) { std::free(ev); return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *out) { *out = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipGetSymbolAddress(void **out, const void *symbol) { *out = const_cast<void *>(symbol); return hipSuccess; }
