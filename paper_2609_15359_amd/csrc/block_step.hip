// Block tables and slots of one decode step: blocks of finished requests go
// back to the ring of free blocks, growing requests take blocks from its
// front, and every new token gets its slot in the cache.
//
// Everything follows from three prefix sums over the request slots (blocks
// that come back, blocks needed, tokens).  They are cheap (12 bytes a slot)
// next to a launch, so each workgroup computes them for itself in LDS and one
// launch does the whole step; that works because the call's outputs never
// overlap its inputs and a block that comes back is not handed out before the
// next call.  Slots are computed per token, two a thread, from per-slot state
// in LDS, and the token that starts a block writes its table entry.  Finished
// rows are moved by one wavefront each, which reads a row before it rewrites
// it.  64 slots of one step: 5.4 us, a chain of loads, two scans and a search;
// 4,096 slots filled with 7.2 M prompt tokens: 35 us, of which 58 MB of slots
// written take 13.
#include "maps_internal.hpp"

namespace maps {
namespace {

struct StepArgs {
    int32_t B, max_blocks, block_size, shift, num_blocks;   // shift: log2(block_size), -1 if no power of two
    const uint8_t* done;
    const int32_t *grow, *lens, *held;
    int32_t *table, *ring;
    const int32_t* ring_pos;
    int32_t *lens_out, *held_out, *ring_pos_out;
    int64_t *tok_off, *slots;
    int64_t T;
    int64_t stretch;                                        // tokens of a wavefront, a multiple of 128
    uint8_t* granted;
    uint32_t* dev_err;
    bool pairs;                                             // slots lie on 16 bytes
};

struct Slot {               // one request slot as the step sees it
    int32_t len, grow, held, back, need;
    bool fits, ended;       // within max_blocks; its request ended
    uint32_t err;
};

__device__ inline uint32_t div_block(const StepArgs& a, uint32_t x) {
    return a.shift >= 0 ? x >> a.shift : x / uint32_t(a.block_size);
}

__device__ inline Slot load_slot(const StepArgs& a, int32_t b) {
    Slot s;
    s.len = a.lens[b];
    s.grow = a.grow[b];
    s.held = a.held[b];
    s.err = 0;
    if (s.len < 0 || s.grow < 0) s.err |= MAPS_ERR_NEG_LEN;
    if (s.held < 0 || s.held > a.max_blocks) s.err |= MAPS_ERR_BLOCK_TABLE;
    s.len = s.len > 0 ? s.len : 0;
    s.grow = s.grow > 0 ? s.grow : 0;
    s.held = s.held < 0 ? 0 : s.held > a.max_blocks ? a.max_blocks : s.held;
    s.back = 0;
    s.ended = a.done && a.done[b];
    if (s.ended) {
        s.back = s.held;
        s.held = s.len = 0;
    }
    const uint32_t len = uint32_t(s.len) + uint32_t(s.grow);      // both are below 2^31
    const uint32_t whole = div_block(a, len), want = whole + (len > whole * uint32_t(a.block_size));
    // (tokens without a block would need blocks that no new token starts)
    s.fits = want <= uint32_t(a.max_blocks) && len <= uint32_t(INT32_MAX) &&
             uint64_t(s.len) <= uint64_t(s.held) * uint32_t(a.block_size);
    if (!s.fits) s.err |= MAPS_ERR_BLOCK_TABLE;
    s.need = s.fits && int32_t(want) > s.held ? int32_t(want) - s.held : 0;
    return s;
}

constexpr uint32_t kFlag = 0x80000000u;

template <int NT>
__global__ __launch_bounds__(NT, 4) void block_step_kernel(StepArgs a) {
    // per slot, 16 bytes: tokens before it, blocks needed before it, its length (kFlag: refused), and its held blocks
    // or, if its request ended (kFlag), the blocks that come back before it
    extern __shared__ __attribute__((aligned(16))) char smem[];
    int32_t* off = reinterpret_cast<int32_t*>(smem);
    int32_t* need = off + a.B + 1;
    uint32_t* len = reinterpret_cast<uint32_t*>(need + a.B + 1);
    uint32_t* own = len + a.B;
    __shared__ int64_t tmp[NT / kWave];
    __shared__ int32_t tmp32[NT / kWave];
    const int tid = threadIdx.x;
    uint32_t head = uint32_t(a.ring_pos[0]), count = uint32_t(a.ring_pos[1]);

    // the slots as they are: growth, blocks needed (kFlag: more than a row takes), length, blocks held or given back
    uint32_t err = 0;
    for (int32_t b = tid; b < a.B; b += NT) {
        const Slot s = load_slot(a, b);
        err |= s.err;
        off[b] = s.grow;
        need[b] = s.need | (s.fits ? 0 : int32_t(kFlag));
        len[b] = uint32_t(s.len);
        own[b] = s.ended ? uint32_t(s.back) | kFlag : uint32_t(s.held);
    }
    __syncthreads();
    // their prefix sums, a run of slots a thread; needed and returned blocks are below 2^31 each and share a word
    const int32_t run = (a.B + NT - 1) / NT, b0 = tid * run, b1 = b0 + run < a.B ? b0 + run : a.B;
    int64_t tokens = 0, blocks = 0;
    auto moves = [&](int32_t b) {
        return int64_t(own[b] & kFlag ? own[b] & ~kFlag : 0) << 32 | (uint32_t(need[b]) & ~kFlag);
    };
    for (int32_t b = b0; b < b1; ++b) {
        tokens += off[b];
        blocks += moves(b);
    }
    int64_t total, moved;
    tokens = block_excl_scan<NT, false, int64_t>(tokens, 0, tmp, &total);
    blocks = block_excl_scan<NT, false, int64_t>(blocks, 0, tmp, &moved);
    const int32_t returned = int32_t(moved >> 32);
    const uint32_t N = uint32_t(a.num_blocks);
    if (head >= N || count > N) {
        err |= MAPS_ERR_BLOCK_TABLE;
        head = count = 0;
    }
    const bool room = uint32_t(returned) <= N - count;   // else the ring has been given blocks twice
    if (!room) err |= MAPS_ERR_BLOCK_TABLE;
    // a token past T would leave the table without the block that it starts: nothing grows then, and no block is lost
    const bool listed = total <= a.T;
    if (!listed) err |= MAPS_ERR_SEG_OFFSETS;
    auto sat = [](int64_t x) { return int32_t(x < INT32_MAX ? x : INT32_MAX); };   // T is no more
    auto at = [&](uint32_t i) { return i >= N ? i - N : i; };                       // i < 2 N
    const bool first_wg = blockIdx.x == 0;
    int32_t took = 0;
    for (int32_t b = b0; b < b1; ++b) {
        const int32_t before = int32_t(blocks), mine = need[b] & int32_t(~kFlag), grow = off[b];
        const int64_t step = moves(b);
        const uint32_t ended = own[b] & kFlag;
        const bool granted = listed && need[b] >= 0 && (mine == 0 || uint32_t(before) + uint32_t(mine) <= count);
        if (first_wg) {
            a.granted[b] = granted;
            a.lens_out[b] = int32_t(len[b]) + (granted ? grow : 0);
            a.held_out[b] = (ended ? 0 : int32_t(own[b])) + (granted ? mine : 0);
            a.tok_off[b] = tokens;
        }
        off[b] = sat(tokens);
        need[b] = before;
        len[b] |= granted ? 0 : kFlag;
        if (ended) own[b] = uint32_t(blocks >> 32) | kFlag;
        if (granted && mine > 0) took = before + mine;
        tokens += grow;
        blocks += step;
    }
    if (tid == 0) {
        off[a.B] = sat(total);
        need[a.B] = int32_t(moved);
        if (first_wg) a.tok_off[a.B] = total;
    }
    __syncthreads();

    // rows of finished requests, and what such a slot takes anew: one wavefront a request, the old row read first
    const int lane = tid & (kWave - 1);
    const int32_t waves = int32_t(gridDim.x) * (NT / kWave);
    if (a.done)
        for (int32_t b = int32_t(blockIdx.x) * (NT / kWave) + tid / kWave; b < a.B; b += waves) {
            const uint32_t mine = own[b];
            if (!(mine & kFlag)) continue;
            int32_t* row = a.table + int64_t(b) * a.max_blocks;
            const int32_t back = a.held[b] < 0 ? 0 : a.held[b] > a.max_blocks ? a.max_blocks : a.held[b];
            if (room)
                for (int32_t j = lane; j < back; j += kWave)
                    a.ring[at(at(head + count) + (mine & ~kFlag) + uint32_t(j))] = row[j];
            const int32_t n = len[b] & kFlag ? 0 : need[b + 1] - need[b];
            for (int32_t j = lane; j < n; j += kWave) row[j] = a.ring[at(head + uint32_t(need[b]) + uint32_t(j))];
        }

    // the slots: a wavefront takes a stretch of tokens, two neighbours a lane and round.  Each lane finds its first
    // token's slot by binary search and walks on from there.
    const int64_t tokens_in = total < a.T ? total : a.T;
    const int64_t from = (int64_t(blockIdx.x) * (NT / kWave) + tid / kWave) * a.stretch;
    const int64_t to = from + a.stretch < a.T ? from + a.stretch : a.T;
    int32_t b = 0;
    if (from + 2 * lane < tokens_in) {
        int32_t hi = a.B - 1;                                         // the last b with off[b] <= t
        while (b < hi) {
            const int32_t mid = (b + hi + 1) >> 1;
            if (off[mid] <= int32_t(from) + 2 * lane) b = mid; else hi = mid - 1;
        }
    }
    for (int64_t t = from + 2 * lane; t < to; t += 2 * kWave) {
        int64_t slot[2] = {-1, -1};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (t + i >= tokens_in) continue;
            while (off[b + 1] <= int32_t(t) + i) ++b;
            const uint32_t start = len[b];
            if (start & kFlag) continue;
            const uint32_t pos = start + uint32_t(int32_t(t) + i - off[b]), j = div_block(a, pos);
            const bool ended = own[b] & kFlag;
            const uint32_t held = ended ? 0 : own[b];
            const int32_t id = j < held ? a.table[int64_t(b) * a.max_blocks + j]
                                        : a.ring[at(head + uint32_t(need[b]) + j - held)];
            const uint32_t place = pos - j * uint32_t(a.block_size);
            if (uint32_t(id) >= N) err |= MAPS_ERR_BLOCK_TABLE;
            else slot[i] = int64_t(id) * a.block_size + place;
            // a block's first token brings it into the table
            if (place == 0 && j >= held && !ended) a.table[int64_t(b) * a.max_blocks + j] = id;
        }
        if (a.pairs && t + 1 < a.T) {
            *reinterpret_cast<longlong2*>(a.slots + t) = longlong2{slot[0], slot[1]};
        } else {
            a.slots[t] = slot[0];
            if (t + 1 < to) a.slots[t + 1] = slot[1];
        }
    }

    if (first_wg) {
        took = block_reduce_max<NT>(took, tmp32);
        if (tid == 0) {
            a.ring_pos_out[0] = int32_t(at(head + uint32_t(took)));
            a.ring_pos_out[1] = int32_t(count - uint32_t(took) + (room ? uint32_t(returned) : 0));
        }
    }
    if (err) raise_error(a.dev_err, err);
}

template <int NT>
void launch(StepArgs a, hipStream_t stream) {
    const size_t lds = size_t(a.B + 1) * 4 * sizeof(int32_t);
    allow_dynamic_lds(block_step_kernel<NT>, lds);
    // two requests a wavefront and 128 tokens, or as many of either as fill the chip
    constexpr int kW = NT / kWave;
    const int64_t most = int64_t(device_compute_units()) * (NT == 256 ? 4 : 1);
    int64_t wgs = (a.B + 2 * kW - 1) / (2 * kW);
    const int64_t for_tokens = (a.T + kW * 2 * kWave - 1) / (kW * 2 * kWave);
    if (for_tokens > wgs) wgs = for_tokens;
    if (wgs > most) wgs = most;
    a.stretch = ((a.T + wgs * kW - 1) / (wgs * kW) + 2 * kWave - 1) / (2 * kWave) * (2 * kWave);
    hipLaunchKernelGGL((block_step_kernel<NT>), dim3(uint32_t(wgs)), dim3(NT), lds, stream, a);
}

}  // namespace
}  // namespace maps

using namespace maps;

extern "C" maps_status maps_block_step(int32_t B, int32_t max_blocks, int32_t block_size, int32_t num_blocks,
                                       const uint8_t* done, const int32_t* grow, const int32_t* lens,
                                       const int32_t* held, int32_t* table, int32_t* ring, const int32_t* ring_pos,
                                       int32_t* lens_out, int32_t* held_out, int32_t* ring_pos_out,
                                       int64_t* tok_off, int64_t* slots, int64_t T, uint8_t* granted,
                                       uint32_t* dev_err, hipStream_t stream) {
    if (B < 1 || B > MAPS_MAX_STEP_REQUESTS || max_blocks < 1 || block_size < 1 || num_blocks < 1 ||
        int64_t(B) * max_blocks > INT32_MAX || T < 0 || T > INT32_MAX)
        return MAPS_E_SIZE;
    if (!grow || !lens || !held || !table || !ring || !ring_pos || !lens_out || !held_out || !ring_pos_out ||
        !tok_off || (T > 0 && !slots) || !granted || !dev_err)
        return MAPS_E_NULL;
    StepArgs a{};
    a.B = B;
    a.max_blocks = max_blocks;
    a.block_size = block_size;
    a.shift = (block_size & (block_size - 1)) == 0 ? __builtin_ctz(unsigned(block_size)) : -1;
    a.num_blocks = num_blocks;
    a.done = done;
    a.grow = grow;
    a.lens = lens;
    a.held = held;
    a.table = table;
    a.ring = ring;
    a.ring_pos = ring_pos;
    a.lens_out = lens_out;
    a.held_out = held_out;
    a.ring_pos_out = ring_pos_out;
    a.tok_off = tok_off;
    a.slots = slots;
    a.T = T;
    a.granted = granted;
    a.dev_err = dev_err;
    a.pairs = reinterpret_cast<uintptr_t>(slots) % 16 == 0;
    // a thread of the prefix sums takes one slot, or few of them with the largest workgroup
    if (B <= 256) launch<256>(a, stream);
    else launch<1024>(a, stream);
    MAPS_CHECK_LAUNCH();
    return MAPS_OK;
}
