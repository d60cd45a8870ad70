// Attention of query tokens over the 4-bit paged cache.
//
// Rows and columns.  The G query heads of a KV head times a request's query
// tokens are columns that share every key and value.  A wavefront holds
// 16 NT columns and walks 32 key positions (a tile) a round, with both
// products on the matrix cores and nothing between them but registers:
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16: a stored key is exact in bf16 and
//                 is converted in registers with its scale; lane (g, r) holds
//                 16 bytes of key r, which are its channels of four steps.  A
//                 query goes in as it is (bf16) or as the sum of two bf16
//                 pieces, which holds all of its bits (f16).  (The scaled 4-bit
//                 instruction needs no conversion, but it drops what lies some
//                 16 bits below the largest product: scores off by 2e-5 of
//                 sum |q||k| in one row of twenty.)
//   O^T += V^T P^T  v_mfma_f32_16x16x32_bf16.  S^T leaves lane (g, c) with
//                 keys 4g..4g+3 of column c, which is the lane of P^T's
//                 operand; the page keeps V in groups of 4 tokens so that one
//                 load gives lane (g, r) the same 4 keys and D / 16 channels,
//                 and conversion by the token's scale plus one byte
//                 permutation gives V^T's.  The probabilities go in as two
//                 bf16 pieces, 16 bits or more; from 32 columns of bf16 queries
//                 on, as one (kPieces below).
// The softmax keeps one running maximum a column, moved only when a score
// exceeds it by 2^8: sums stay far inside 32 bits, and most tiles need no
// exchange between lanes.
//
// Splitting.  All tiles of all (request, KV head, block of columns) lie on
// one line; every wavefront takes the same number of consecutive tiles, so
// ragged lengths, long single requests and many short ones are balanced alike.
// The blocks of columns of a prompt see falling parts of it: the first and the
// last, the second and the one before the last, .. share one stretch.  A
// stretch that is cut leaves partial sums (maximum, sum, products), joined
// first among the wavefronts of a workgroup and then by a second launch, both
// in the order of the line: the same inputs give the same bits.
//
// Measured, us a call (both launches; cards differ by 5%): 256 requests of 128
// .. 8,192 tokens, 8 KV heads of 128, 4 query heads each, bf16: 123 = 4.4 TB/s
// of cache, bound by memory (a large copy runs at 4.8 .. 4.9); one request of
// 131,072 tokens: 44, of which the join is 8; up to 5 drafted tokens a request
// and 6 heads a KV head in f16 with a window: 77, vector instructions 34% of
// the SIMDs' cycles (conversions, and a softmax whose columns are half empty),
// products 26%, the rest waits that two wavefronts a SIMD do not cover; 2,048
// query tokens of two requests of 9,742 and 13,777: 913 .. 970 = 743 .. 789
// TFLOP/s, vector instructions 56%, products 33% (a large matrix product of the
// library reaches 1,190 .. 1,215).
#include "kv_page.hpp"

namespace maps {
namespace {

using kv::f32x4;
using kv::u32x4;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kTile = 32;          // key positions a round
constexpr int kWaves = 4;          // wavefronts of a workgroup
constexpr int kAttendNT = kWaves * kWave;
constexpr int kSetUp = 3;          // what a stretch costs besides its tiles, in tiles
constexpr int kMinTiles = kSetUp + 1;   // shortest share of a wavefront
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct AttendArgs {
    const char* cache;
    int32_t num_blocks, shift, H, Hq, G, B, max_blocks, max_q, window;
    int32_t Q, heads_per, subs;    // a block of columns: Q query tokens of heads_per of the G heads, subs groups of them
    int64_t page, T, q_st, q_sh;
    uint32_t block, v_skip;        // bytes of a block; from a page's keys to its values
    const void* q;
    const int32_t *table, *lens;
    const int64_t* tok_off;
    float scale;
    void* out;
    float* lse;
    uint32_t* dev_err;
    struct Join* joins;            // [workgroups] what the join has to do
    float* parts;                  // [wavefronts][2] partial sums
};

// A stretch of columns that several workgroups share.
struct Join {
    int64_t x0, x1;                // its tiles on the line; x1 = 0: nothing to join
    int64_t per;                   // tiles of one wavefront
    int32_t b, h, c, pad;          // request, KV head, block of columns
};

// Partial sums of 16 NT columns: D products a column, then its maximum and sum.
__host__ __device__ constexpr int64_t part_floats(int cols, int D) { return int64_t(cols) * (D + 2); }

// What a request asks for, from its arrays.
struct Request {
    int32_t len, n;                // tokens, query tokens (the last n)
    int64_t q0;                    // its first row
    uint32_t err;
};

__device__ inline Request request_of(const AttendArgs& a, int32_t len, int64_t q0, int64_t q1) {
    Request r{len, 0, q0, 0};
    const int64_t n = q1 - q0;
    if (r.len < 0) r.err |= MAPS_ERR_NEG_LEN;
    if (r.q0 < 0 || n < 0 || q1 > a.T || n > a.max_q) r.err |= MAPS_ERR_SEG_OFFSETS;
    if ((int64_t(a.max_blocks) << a.shift) < r.len) r.err |= MAPS_ERR_BLOCK_TABLE;
    r.n = r.err ? 0 : int32_t(n);
    return r;
}

// A value that all lanes hold, as a scalar.
__device__ inline int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
    return int64_t(uint64_t(uint32_t(uniform(int32_t(uint64_t(x) >> 32)))) << 32 | uint32_t(uniform(int32_t(x))));
}

// A load whose address all lanes hold, from an array that the kernel does not write: through the scalar cache.
template <typename V>
__device__ inline V scalar_load(const V* p) {
    return *reinterpret_cast<const __attribute__((address_space(4))) V*>(reinterpret_cast<uintptr_t>(p));
}

// x / y of numbers >= 0, in 32 bits where they fit: the long division takes many times as long.
__device__ inline int64_t divide(int64_t x, int64_t y) {
    return (uint64_t(x) | uint64_t(y)) >> 32 ? x / y : int64_t(uint32_t(x) / uint32_t(y));
}

// Blocks of columns of a request, and the tiles that block c sees: [first, first + count), count >= 1.
__device__ inline int col_blocks(const AttendArgs& a, const Request& r) { return (r.n + a.Q - 1) / a.Q; }
struct Span {
    int32_t first, count;
};
__device__ inline Span span_of(const AttendArgs& a, const Request& r, int c) {
    const int32_t base = r.len - r.n;                       // position of query 0; below 0 it sees nothing
    const int32_t last = base + ((c + 1) * a.Q < r.n ? (c + 1) * a.Q : r.n) - 1;
    int64_t low = a.window ? int64_t(base) + c * a.Q - a.window + 1 : 0;  // (base may be far below 0, window 2^31 - 1)
    low = low > 0 ? low : 0;
    const int32_t first = int32_t(low / kTile);
    const int32_t end = int32_t((uint32_t(last) + kTile) / kTile);        // last >= 0: ceil((last + 1) / 32)
    return {first, last >= 0 && end > first ? end - first : 1};
}

// A place on the line.
struct Place {
    int32_t b, h, c;               // request, KV head and group of its heads, block of columns
    int64_t x0;                    // where its tile 0 lies
    Span span;
};

template <int D, int NT, bool F16>
struct Wave {
    static constexpr int kCols = 16 * NT;
    static constexpr int kSteps = D / 32;                             // 32-channel steps of the scores
    static constexpr int kTerms = F16 ? 2 : 1;                        // bf16 pieces of a query
    // bf16 pieces of a probability.  One leaves an error against 64 bits that is 1.1 to 1.35 times that of rounding the
    // output alone (2.0e-3 .. 2.3e-3 of the outputs' norm against 1.6e-3 .. 1.8e-3), two leave no more than that.  With 16
    // columns, where memory bounds, two take 125.0 us instead of 123.9 (256 requests), 39.4 instead of 39.1 (one of
    // 131,072 positions); in prompts, which the products bound, 1,128 instead of 906 (2,048 query tokens of two
    // requests): there one is enough for outputs of the same 8 bits.
    static constexpr int kPieces = F16 || NT == 1 ? 2 : 1;
    static constexpr int kChunks = D > 128 ? D / 128 : 1;              // scales of a lane's channels of a key
    static constexpr int kOut = D / 16;                               // 16-channel steps of the output
    static constexpr int kBytes = D / 32;                             // V bytes of a lane and token
    using T = typename std::conditional<F16, _Float16, __bf16>::type;

    struct Tile {
        uint32_t k[2][kSteps];
        uint32_t ks[2][kChunks];
        uint32_t none[2];          // scale bits of a half whose block does not exist: NaN, else 0
        uint32_t v[2][kBytes];
        uint32_t vs[2];
    };

    const AttendArgs& a;
    const int lane, g, r;          // lane = 16 g + r
    bool bad = false;              // a block id was out of range

    u32x4 q[NT][kTerms][kSteps];   // queries
    f32x4 acc[NT][kOut];           // O^T: lane (g, column r) holds channels g D/4 .. of its column
    float m[NT], l[NT];            // maximum so far (in powers of two), this lane's part of the sum
    int32_t pos[NT];               // position of the column's query, -1 if it sees nothing

    // of the current stretch
    Tile held;                     // the tile in registers or under way
    const int32_t* row;            // block table
    const char* pages;             // the KV head's page of block 0
    int32_t len;

    __device__ Wave(const AttendArgs& a_) : a(a_), lane(threadIdx.x % kWave), g(lane / 16), r(lane % 16) {}

    // Column c of a block: its query token and head, or false.
    __device__ bool column(const Request& rq, const Place& p, int c, int64_t* t, int* head) const {
        const int sub = p.h % a.subs;
        const int heads = a.G - sub * a.heads_per < a.heads_per ? a.G - sub * a.heads_per : a.heads_per;
        // c / heads: both are at most 64, so the quotient is off by far less than the half that is added
        const int of = int((float(c) + 0.5f) * __builtin_amdgcn_rcpf(float(heads))), qi = p.c * a.Q + of;
        *t = rq.q0 + qi;
        *head = p.h / a.subs * a.G + sub * a.heads_per + c - of * heads;
        return of < a.Q && qi < rq.n;
    }

    // The first of the 8 channels that this lane brings to a step of the scores.
    __device__ int channel(int step) const {
        return D == 64 ? 16 * g + 8 * step : step / 4 * 128 + 32 * g + step % 4 * 8;
    }

    // What two numbers' rounding to bf16 left, rounded to bf16.
    __device__ static kv::bf16x2 rest(float x, float y, kv::bf16x2 hi) {
        const uint32_t w = __builtin_bit_cast(uint32_t, hi);
        return kv::bf16x2{__bf16(x - __uint_as_float(w << 16)), __bf16(y - __uint_as_float(w & 0xffff0000u))};
    }

    // The queries of one block of columns.
    __device__ void load_queries(const Request& rq, const Place& p) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            int64_t t;
            int head;
            const bool live = column(rq, p, nt * 16 + r, &t, &head);
            pos[nt] = live ? rq.len - rq.n + int32_t(t - rq.q0) : -1;
            m[nt] = -INFINITY;
            l[nt] = 0.0f;
#pragma unroll
            for (int j = 0; j < kOut; ++j) acc[nt][j] = f32x4{0, 0, 0, 0};
            const T* src = static_cast<const T*>(a.q) + t * a.q_st + head * a.q_sh;
            // a scale below 0 turns the queries, so that the largest score is the largest product
            const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                u32x4 x = {0, 0, 0, 0};
                if (live) x = *reinterpret_cast<const u32x4*>(src + channel(i)) ^ flip;
                if constexpr (F16) {
                    // 11 bits: 8 rounded to the nearest, which leaves at most 3 and a sign
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t two = x[k];
                        const kv::f16x2 y = __builtin_bit_cast(kv::f16x2, two);
                        const kv::bf16x2 hi = {__bf16(float(y[0])), __bf16(float(y[1]))};
                        const kv::bf16x2 lo = rest(float(y[0]), float(y[1]), hi);
                        q[nt][0][i][k] = __builtin_bit_cast(uint32_t, hi);
                        q[nt][kTerms - 1][i][k] = __builtin_bit_cast(uint32_t, lo);
                    }
                } else {
                    q[nt][0][i] = x;
                }
            }
        }
    }

    // A reduction over the four lanes 16 g + r of a column.
    template <typename V, typename F>
    __device__ static V over_groups(V x, F f) {
        // swapping x's odd rows of 16 (then its upper 32 lanes) with its even ones (lower) leaves both in each lane
        const auto u = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x),
                                                        false, false);
        x = f(__builtin_bit_cast(V, uint32_t(u[0])), __builtin_bit_cast(V, uint32_t(u[1])));
        const auto v = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x),
                                                        false, false);
        return f(__builtin_bit_cast(V, uint32_t(v[0])), __builtin_bit_cast(V, uint32_t(v[1])));
    }

    // The blocks that hold a tile's two halves; the second half may lie past the request: then it is the first's.
    struct Ids {
        int32_t id[2];
    };
    __device__ Ids load_ids(int32_t tile) const {
        const int32_t t0 = tile * kTile, t1 = t0 + 16 < len ? t0 + 16 : t0;
        return {scalar_load(row + (t0 >> a.shift)), scalar_load(row + (t1 >> a.shift))};
    }

    // Where the halves' keys and key scales lie; the values' are a.v_skip behind them.
    struct Pages {
        const char *code[2], *scale[2];
        uint32_t none[2];
    };
    __device__ Pages pages_of(int32_t tile, Ids ids) {
        Pages p;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int32_t t = tile * kTile + (s && tile * kTile + 16 < len ? 16 : 0);
            uint32_t id = uint32_t(ids.id[s]);
            p.none[s] = 0;
            if (id >= uint32_t(a.num_blocks)) {
                // block 0 is read in its place, as keys that are NaN: so is what a query that sees them gets
                bad = true;
                id = 0;
                p.none[s] = kv::kScaleNan << 23;
            }
            const uint32_t at = uint32_t(t) & ((1u << a.shift) - 1);   // a multiple of 16
            const char* page = pages + uint64_t(id) * a.block;
            p.code[s] = page + at * (D / 2);
            p.scale[s] = page + ((uint32_t(D / 2) << a.shift) + at * (D / 32));
        }
        return p;
    }

    __device__ void load_keys(Tile& w, const Pages& p) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            w.none[s] = p.none[s];
            if constexpr (D == 64) {                                   // 16 channels of the half's key r
                const kv::u32x2 x = *reinterpret_cast<const kv::u32x2*>(p.code[s] + uint32_t(r * (D / 2) + g * 8));
                w.k[s][0] = x[0];
                w.k[s][1] = x[1];
                w.ks[s][0] = uint8_t(p.scale[s][uint32_t(r * (D / 32) + g / 2)]);
            } else {
#pragma unroll
                for (int c = 0; c < kChunks; ++c) {                    // 32 of every 128 channels
                    const u32x4 x = *reinterpret_cast<const u32x4*>(p.code[s] + uint32_t(r * (D / 2) + (c * 4 + g) * 16));
#pragma unroll
                    for (int i = 0; i < 4; ++i) w.k[s][c * 4 + i] = x[i];
                    w.ks[s][c] = uint8_t(p.scale[s][uint32_t(r * (D / 32) + c * 4 + g)]);
                }
            }
        }
    }

    __device__ void load_values(Tile& w, const Pages& p) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int i = 0; i < kBytes; ++i)
                w.v[s][i] = *reinterpret_cast<const uint32_t*>(p.code[s] + a.v_skip + uint32_t(lane * (D / 8) + i * 4));
            w.vs[s] = *reinterpret_cast<const uint32_t*>(p.scale[s] + a.v_skip +
                                                         uint32_t(g * (D / 8) + r * D / 512 * 4));
        }
    }

    __device__ bool sees(int nt, int32_t t) const {
        return t <= pos[nt] && (!a.window || t > pos[nt] - a.window);
    }

    // One tile.  edge: some column may not see all of it.  The keys of the tile that is to be held in its place are
    // asked for as soon as its own are used, and the values likewise.
    __device__ __forceinline__ void step(Tile& w, int32_t tile, float c, const Pages& next, bool edge) {
        const int32_t t0 = tile * kTile;
        uint32_t nan = 0;          // V scales that are NaN, a bit a half and token, of this lane's keys
        uint32_t p[NT][kPieces][4];
        float t[NT][8];            // raw scores; the powers of two are c times them
        auto highest = [&](int nt) {
            float top = t[nt][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, t[nt][i]);
            return top * c;
        };
        bool grow = false;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            f32x4 z[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) z[nt] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const float scale = __uint_as_float(w.ks[s][D == 64 ? 0 : i / 4] << 23 | w.none[s]);
                u32x4 k;
                unrolled<4>([&](auto byte) {
                    constexpr int b = decltype(byte)::value;
                    k[b] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w.k[s][i], scale, b));
                });
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < kTerms; ++e)
                        z[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k),
                                                                        __builtin_bit_cast(bf16x8, q[nt][e][i]), z[nt], 0, 0, 0);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) t[nt][4 * s + i] = z[nt][i];
        }
        load_keys(w, next);
        if (edge) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (!sees(nt, t0 + 16 * (i / 4) + 4 * g + i % 4)) t[nt][i] = -INFINITY;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            grow |= highest(nt) > m[nt] + 8.0f;
        }
        if (__any(grow)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float top = fmaxf(m[nt], over_groups(highest(nt), [](float u, float v) { return fmaxf(u, v); }));
                const float fix = top == m[nt] ? 1.0f : __builtin_amdgcn_exp2f(m[nt] - top);
                m[nt] = top;
                l[nt] *= fix;
#pragma unroll
                for (int j = 0; j < kOut; ++j) acc[nt][j] *= fix;
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float base = m[nt] == -INFINITY ? 0.0f : m[nt];
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(t[nt][i], c, -base));
                l[nt] += e[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const kv::bf16x2 hi = {__bf16(e[2 * i]), __bf16(e[2 * i + 1])};
                p[nt][0][i] = __builtin_bit_cast(uint32_t, hi);
                if constexpr (kPieces == 2) {
                    const kv::bf16x2 lo = rest(e[2 * i], e[2 * i + 1], hi);
                    p[nt][1][i] = __builtin_bit_cast(uint32_t, lo);
                }
            }
        }
        if (edge) {
            // values past the request are unset, and a NaN must not reach columns that do not see its position:
            // both become zeros here, the visible ones are put back below
#pragma unroll
            for (int s = 0; s < 2; ++s) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool past = t0 + 16 * s + 4 * g + i >= len;
                    const bool is_nan = (w.vs[s] >> 8 * i & 255) == kv::kScaleNan;
                    if (past || is_nan) w.vs[s] = (w.vs[s] & ~(255u << 8 * i)) | kv::kScaleOne << 8 * i;
                    if (is_nan && !past) nan |= 1u << (4 * s + i);
                    if (past || is_nan) {
                        // token i's kBytes bytes
#pragma unroll
                        for (int e = 0; e < kBytes; ++e)
                            w.v[s][(i * kBytes + e) / 4] &= ~(255u << 8 * ((i * kBytes + e) % 4));
                    }
                }
            }
        }
        float vscale[2][4];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) vscale[s][i] = kv::scale_value(w.vs[s] >> 8 * i & 255);
        unrolled<kBytes>([&](auto byte) {
            constexpr int b = decltype(byte)::value;                   // channels 2 b and 2 b + 1 of the lane's
            uint32_t two[2][4];
            unrolled<4>([&](auto token) {
                constexpr int i = decltype(token)::value, flat = i * kBytes + b;
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    two[s][i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(
                                                                 w.v[s][flat / 4], vscale[s][i], flat % 4));
            });
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t sel = half ? 0x07060302u : 0x05040100u;
                const u32x4 va = {__builtin_amdgcn_perm(two[0][1], two[0][0], sel),
                                  __builtin_amdgcn_perm(two[0][3], two[0][2], sel),
                                  __builtin_amdgcn_perm(two[1][1], two[1][0], sel),
                                  __builtin_amdgcn_perm(two[1][3], two[1][2], sel)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int k = 0; k < kPieces; ++k) {
                        const u32x4 pb = {p[nt][k][0], p[nt][k][1], p[nt][k][2], p[nt][k][3]};
                        acc[nt][2 * b + half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, va), __builtin_bit_cast(bf16x8, pb), acc[nt][2 * b + half], 0, 0, 0);
                    }
            }
        });
        load_values(w, next);
        if (edge && __any(nan != 0)) spread_nan(nan, t0);
    }

    // NaN scales of an edge tile (bits as in step, lane (g', r') holding channels r' D/16..) onto the outputs of the
    // columns that see them: lane (g, r) holds channels g D/4 .. +D/4 of column r.
    __device__ void spread_nan(uint32_t nan, int32_t t0) {
        float add[NT][D > 128 ? 2 : 1] = {};
#pragma unroll 1
        for (int k = 0; k < kTile; ++k) {                                       // key t0 + k: lane group k % 16 / 4
#pragma unroll
            for (int part = 0; part < (D > 128 ? 2 : 1); ++part) {
                const int block = D > 128 ? 2 * g + part : g * (D / 4) / 32;   // 32 channels of this lane
                const uint32_t bits = uint32_t(__shfl(int(nan), 16 * (k % 16 / 4) + block * 512 / D, kWave));
                const bool is_nan = bits >> (4 * (k / 16) + k % 4) & 1;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) add[nt][part] = is_nan && sees(nt, t0 + k) ? NAN : add[nt][part];
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < kOut; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nt][j][i] += add[nt][D > 128 ? i / 2 : 0];
    }

    template <int N, typename F, int I = 0>
    __device__ static void unrolled(F f) {
        if constexpr (I < N) {
            f(std::integral_constant<int, I>{});
            unrolled<N, F, I + 1>(f);
        }
    }

    // Tiles [first, end) of a stretch, of the tiles that the columns see.
    __device__ void walk(const Request& rq, const Place& p, int32_t first, int32_t end) {
        first = uniform(first);
        end = uniform(end);
        len = rq.len;
        row = a.table + int64_t(p.b) * a.max_blocks;
        pages = a.cache + int64_t(p.h / a.subs) * a.page;
        const int32_t lo = rq.len - rq.n + p.c * a.Q;                  // the block's first and last query position
        const int32_t hi = rq.len - rq.n + ((p.c + 1) * a.Q < rq.n ? (p.c + 1) * a.Q : rq.n) - 1;
        if (hi < 0) {                                                  // nothing is seen, nothing is there to read
            load_queries(rq, p);
            return;
        }
        // the first tile is on its way while the queries are laid out; behind the last tile it is asked for again, which
        // keeps the rounds free of branches.  (Two tiles in registers: 256 requests 125 us instead of 121.)
        auto clip = [&](int32_t tile) { return tile < end ? tile : end - 1; };
        {
            const Pages to = pages_of(first, load_ids(first));
            load_keys(held, to);
            load_values(held, to);
        }
        Ids ids = load_ids(clip(first + 1));
        load_queries(rq, p);
        // a scale of zero would make NaN of the infinities that mark unseen positions: 2^-149 stands for it, which leaves
        // 2^-21 of the largest finite product
        const float c = a.scale == 0.0f ? 0x1p-149f : fabsf(a.scale) * kLog2e;
        for (int32_t tile = first; tile < end; ++tile) {
            const bool edge = tile * kTile + kTile - 1 > lo || (a.window && tile * kTile <= hi - a.window);
            const Pages to = pages_of(clip(tile + 1), ids);
            ids = load_ids(clip(tile + 2));
            step(held, tile, c, to, edge);
        }
    }

    // The column's whole sum, of the lanes' parts.
    __device__ float sum(int nt) const {
        return over_groups(l[nt], [](float u, float v) { return u + v; });
    }

    __device__ void store_part(float* part) const {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float total = sum(nt);
            if (pos[nt] < 0) continue;                                 // no column, or one that sees nothing
            float* col = part + (nt * 16 + r) * D + g * (D / 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < kOut; j += 4)
                    *reinterpret_cast<f32x4*>(col + i * kOut + j) =
                        f32x4{acc[nt][j][i], acc[nt][j + 1][i], acc[nt][j + 2][i], acc[nt][j + 3][i]};
            if (g == 0) {
                part[kCols * D + nt * 16 + r] = m[nt];
                part[kCols * (D + 1) + nt * 16 + r] = total;
            }
        }
    }

    // Adds a stored part of later tiles; afterwards l is the whole sum, held in group 0.
    __device__ void add_part(const float* part) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (pos[nt] < 0) continue;
            const float m2 = part[kCols * D + nt * 16 + r], l2 = g == 0 ? part[kCols * (D + 1) + nt * 16 + r] : 0.0f;
            const float top = fmaxf(m[nt], m2);
            const float f1 = top == m[nt] ? 1.0f : __builtin_amdgcn_exp2f(m[nt] - top);
            const float f2 = top == m2 ? 1.0f : __builtin_amdgcn_exp2f(m2 - top);
            m[nt] = top;
            l[nt] = l[nt] * f1 + l2 * f2;
            const float* col = part + (nt * 16 + r) * D + g * (D / 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < kOut; j += 4) {
                    const f32x4 v = *reinterpret_cast<const f32x4*>(col + i * kOut + j);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[nt][j + k][i] = acc[nt][j + k][i] * f1 + v[k] * f2;
                }
        }
    }

    __device__ void finish(const Request& rq, const Place& p) const {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float total = sum(nt);
            int64_t t;
            int head;
            if (!column(rq, p, nt * 16 + r, &t, &head)) continue;
            const bool none = pos[nt] < 0;
            const float inv = none ? 0.0f : 1.0f / total;
            T* dst = static_cast<T*>(a.out) + (t * a.Hq + head) * D + g * (D / 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                T e[kOut];
#pragma unroll
                for (int j = 0; j < kOut; ++j) e[j] = T(none ? 0.0f : acc[nt][j][i] * inv);
                if constexpr (kOut == 4) {
                    *reinterpret_cast<kv::u32x2*>(dst + i * kOut) = *reinterpret_cast<kv::u32x2*>(e);
                } else {
#pragma unroll
                    for (int k = 0; k < kOut / 8; ++k)
                        reinterpret_cast<u32x4*>(dst + i * kOut)[k] = reinterpret_cast<u32x4*>(e)[k];
                }
            }
            if (a.lse && g == 0) a.lse[t * a.Hq + head] = none ? -INFINITY : (m[nt] + __builtin_amdgcn_logf(total)) * kLn2;
        }
    }
};

// Where tile x of the line lies.  off[b]: the tiles before request b.  false: x lies in the gap that a pair of blocks
// of columns leaves; *next is then the first tile behind it.
__device__ inline bool place_of(const AttendArgs& a, const int64_t* off, int64_t x, Place* p, Request* rq,
                                int32_t* tile, int64_t* next) {
    int32_t lo = 0, hi = a.B;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (off[mid] <= x) lo = mid; else hi = mid;
    }
    lo = uniform(lo);
    p->b = lo;
    *rq = request_of(a, scalar_load(a.lens + lo), scalar_load(a.tok_off + lo), scalar_load(a.tok_off + lo + 1));
    const int blocks = col_blocks(a, *rq), pairs = (blocks + 1) / 2;
    const int64_t before = uniform(off[lo]);
    const int64_t stretch = divide(uniform(off[lo + 1]) - before, int64_t(a.H) * a.subs * pairs), in = x - before;
    const int64_t at = divide(in, stretch);
    const int32_t u = int32_t(in - at * stretch);
    p->h = int32_t(divide(at, pairs));
    const int pair = int32_t(at - int64_t(p->h) * pairs);
    p->c = pair;
    p->span = span_of(a, *rq, pair);
    p->x0 = x - u;
    *tile = u;
    if (u < p->span.count) return true;
    *next = x - u + stretch;
    if (blocks - 1 - pair == pair) return false;
    const int32_t skip = p->span.count;
    p->c = blocks - 1 - pair;
    p->span = span_of(a, *rq, p->c);
    p->x0 += skip;
    *tile = u - skip;
    return *tile < p->span.count;
}

template <int D, int NT, bool F16>
constexpr int attend_waves() { return NT == 1 && D <= 128 ? 3 : NT * D <= 256 ? 2 : 1; }

template <int D, int NT, bool F16>
__global__ __launch_bounds__(kAttendNT, (attend_waves<D, NT, F16>())) void kv_attend_kernel(AttendArgs a) {
    using W = Wave<D, NT, F16>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    int64_t* off = reinterpret_cast<int64_t*>(smem);                 // [B + 1]
    __shared__ int64_t tmp[kWaves];
    const int tid = threadIdx.x, wid = __builtin_amdgcn_readfirstlane(tid / kWave);

    uint32_t err = 0;
    for (int32_t b = tid; b < a.B; b += kAttendNT) {
        const Request r = request_of(a, a.lens[b], a.tok_off[b], a.tok_off[b + 1]);
        err |= r.err;
        const int blocks = col_blocks(a, r), pairs = (blocks + 1) / 2;
        int64_t stretch = 0;                                         // the longest pair of blocks of columns
        for (int c = 0; c < pairs; ++c) {
            const int other = blocks - 1 - c;
            const int64_t n = span_of(a, r, c).count + (other != c ? span_of(a, r, other).count : 0);
            stretch = n > stretch ? n : stretch;
        }
        off[b] = (stretch + kSetUp) * pairs * a.H * a.subs;
    }
    __syncthreads();
    const int64_t total = block_scan<kAttendNT, false, false, true, int64_t>(
        a.B, 0, [&](int64_t i) { return off[i]; }, [&](int64_t i, int64_t v) { off[i] = v; }, tmp);
    if (tid == 0) off[a.B] = total;
    __syncthreads();

    // rows past the last request
    {
        const int64_t from = a.tok_off[a.B] < 0 ? a.T : a.tok_off[a.B];
        using T = typename W::T;
        for (int64_t i = from * a.Hq * D + int64_t(blockIdx.x) * kAttendNT + tid; i < a.T * a.Hq * D;
             i += int64_t(gridDim.x) * kAttendNT) {
            static_cast<T*>(a.out)[i] = T(0.0f);
            if (a.lse && i % D == 0) a.lse[i / D] = -INFINITY;
        }
    }

    const int64_t waves = int64_t(gridDim.x) * kWaves;
    int64_t per = divide(uniform(total) + waves - 1, waves);
    per = uniform(per > kMinTiles ? per : kMinTiles);
    const int64_t wave = int64_t(blockIdx.x) * kWaves + wid;
    const int64_t start = wave * per, end = start + per < uniform(total) ? start + per : uniform(total);
    const int64_t wg_start = int64_t(blockIdx.x) * kWaves * per, wg_end = wg_start + kWaves * per;
    const int64_t part = part_floats(W::kCols, D);

    W w(a);
    Place p{};
    Request rq{};
    int64_t x = start, open = 0;                // open: end on the line of a last stretch that goes on behind this wavefront
    Join join{};
    while (x < end) {
        int32_t tile;
        int64_t next = 0;
        const bool there = place_of(a, off, x, &p, &rq, &tile, &next);
        tile = uniform(tile);
        next = uniform(next);
        p = Place{uniform(p.b), uniform(p.h), uniform(p.c), uniform(p.x0), {uniform(p.span.first), uniform(p.span.count)}};
        rq = Request{uniform(rq.len), uniform(rq.n), uniform(rq.q0), 0};
        if (!uniform(int32_t(there))) {
            x = next;
            continue;
        }
        const int32_t left = p.span.count - tile, n = end - x < left ? int32_t(end - x) : left;
        w.walk(rq, p, p.span.first + tile, p.span.first + tile + n);
        const int64_t x1 = p.x0 + p.span.count;
        if (tile == 0 && n == p.span.count) {
            w.finish(rq, p);
        } else {
            w.store_part(a.parts + (wave * 2 + (x == start ? 0 : 1)) * part);
            if (x + n < x1) open = x1;
            // the first workgroup border inside the stretch has it joined
            if (wid == 0 && x == start && p.x0 < wg_start && p.x0 >= wg_start - kWaves * per)
                join = Join{p.x0, x1, per, p.b, p.h, p.c, 0};
        }
        x = uniform(x + n);
    }
    if (wid == 0 && tid == 0) a.joins[blockIdx.x] = join;
    if (w.bad) err |= MAPS_ERR_BLOCK_TABLE;
    if (err) raise_error(a.dev_err, err);

    // stretches cut inside the workgroup: the first of their wavefronts adds the others' parts to its own
    __syncthreads();
    if (!open || !(p.x0 >= start || wid == 0)) return;
    const int64_t slot = (wave * 2 + (p.x0 > start ? 1 : 0)) * part;
    bool added = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const float whole = w.sum(nt);
        w.l[nt] = w.g == 0 ? whole : 0.0f;
    }
    for (int64_t i = wave + 1; i < int64_t(blockIdx.x + 1) * kWaves && i * per < open; ++i) {
        w.add_part(a.parts + i * 2 * part);
        added = true;
    }
    if (p.x0 >= wg_start && open <= wg_end) w.finish(rq, p);
    else if (added) w.store_part(a.parts + slot);
}

// The parts of a stretch, one from each workgroup that it crosses, in their order.  A thread takes 4 channels of a
// live column (a unit) over every kth part, four parts under way at a time; the k sums are joined in LDS.
constexpr int kJoinNT = 512;
// Where there are so few stretches that most workgroups would find nothing to join, kJoinSplit of them share a
// stretch's units, each with more threads for its parts.  (With many, the further workgroups only cost their start.)
constexpr int kJoinSplit = 4;

struct Sum {
    float m, l;
    f32x4 o;
    __device__ void add(float m2, float l2, f32x4 o2) {
        const float top = fmaxf(m, m2);
        const float f1 = top == m ? 1.0f : __builtin_amdgcn_exp2f(m - top);
        const float f2 = top == m2 ? 1.0f : __builtin_amdgcn_exp2f(m2 - top);
        m = top;
        l = l * f1 + l2 * f2;
        o = o * f1 + o2 * f2;
    }
};

template <int D, int NT, bool F16>
__global__ __launch_bounds__(kJoinNT) void kv_join_kernel(AttendArgs a) {
    using W = Wave<D, NT, F16>;
    using T = typename W::T;
    const Join jn = a.joins[blockIdx.x];
    if (jn.x1 == 0) return;
    constexpr int kCols = W::kCols;
    constexpr int64_t part = part_floats(kCols, D);
    __shared__ Sum sums[kJoinNT];
    const int64_t per4 = jn.per * kWaves, j0 = jn.x0 / per4, j1 = (jn.x1 - 1) / per4;
    const float* lead = a.parts + (jn.x0 / jn.per * 2 + (jn.x0 % jn.per ? 1 : 0)) * part;     // workgroup j0's part
    const Request rq = request_of(a, a.lens[jn.b], a.tok_off[jn.b], a.tok_off[jn.b + 1]);
    const Place p{jn.b, jn.h, jn.c, jn.x0, {}};
    const W w(a);
    const int sub = p.h % a.subs, heads = a.G - sub * a.heads_per < a.heads_per ? a.G - sub * a.heads_per : a.heads_per;
    const int tokens = rq.n - p.c * a.Q < a.Q ? rq.n - p.c * a.Q : a.Q;
    const int all = heads * tokens * (D / 4), share = (all + int(gridDim.y) - 1) / int(gridDim.y);
    const int u_from = int(blockIdx.y) * share, units = all - u_from < share ? all - u_from : share;
    if (units <= 0) return;
    const int groups = units < kJoinNT ? kJoinNT / units : 1, group = groups > 1 ? threadIdx.x / units : 0;
    for (int u0 = 0; u0 < units; u0 += kJoinNT) {
        const int i = groups > 1 ? int(threadIdx.x) - group * units : u0 + int(threadIdx.x), u = u_from + i;
        const bool live = group < groups && i < units;
        const int col = u / (D / 4);
        Sum s{-INFINITY, 0.0f, {0, 0, 0, 0}};
        if (live) {
            constexpr int kDeep = 4;
            for (int64_t j = j0 + group; j <= j1; j += kDeep * groups) {
                float m2[kDeep], l2[kDeep];
                f32x4 o2[kDeep];
#pragma unroll
                for (int k = 0; k < kDeep; ++k) {
                    const int64_t jk = j + k * groups;
                    const float* src = jk == j0 ? lead : a.parts + (jk <= j1 ? jk : j1) * kWaves * 2 * part;
                    m2[k] = jk <= j1 ? src[kCols * D + col] : -INFINITY;
                    l2[k] = jk <= j1 ? src[kCols * (D + 1) + col] : 0.0f;
                    o2[k] = *reinterpret_cast<const f32x4*>(src + u * 4);
                    if (jk > j1) o2[k] = f32x4{0, 0, 0, 0};
                }
#pragma unroll
                for (int k = 0; k < kDeep; ++k) s.add(m2[k], l2[k], o2[k]);
            }
        }
        if (groups > 1) {
            sums[threadIdx.x] = s;
            __syncthreads();
            if (group == 0)
                for (int k = 1; k < groups; ++k) {
                    const Sum& x = sums[threadIdx.x + k * units];
                    s.add(x.m, x.l, x.o);
                }
        }
        int64_t t;
        int head;
        if (!live || group || !w.column(rq, p, col, &t, &head)) continue;
        const bool none = rq.len - rq.n + int32_t(t - rq.q0) < 0;
        T e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = T(none ? 0.0f : s.o[i] / s.l);
        *reinterpret_cast<kv::u32x2*>(static_cast<T*>(a.out) + (t * a.Hq + head) * D + u % (D / 4) * 4) =
            *reinterpret_cast<kv::u32x2*>(e);
        if (a.lse && u % (D / 4) == 0)
            a.lse[t * a.Hq + head] = none ? -INFINITY : (s.m + __builtin_amdgcn_logf(s.l)) * kLn2;
    }
}

// 16-column steps of a wavefront.  More of them share the keys' and values' conversions, until the sums leave the 256
// registers of half the file and are moved between its halves around every branch:
// Measured in bf16 / f16, us, on prompts (the last tokens of two requests of 9,742 and 13,777, 4 heads a KV head) and
// chunks (100 tokens of 16 requests of 500 .. 4,000):
//   64 channels: as few as hold the longest request's columns, at most 4 (1,024 tokens 276 / 399, with 2 377 / 460, although
//   14 registers spill in f16; chunks 69 / 91, with 2 73 / 86);
//   128: at most 2 (2,048 tokens 909 / 1,258, with 4 1,105 / 2,016, with 1 1,384 / 1,596; chunks 95 / 120, with 4 127 / 213);
//   256: 2 (700 tokens 437 / 542, with 1 546 / 570; chunks 121 / 144, with 1 124 / 129), but 1 up to 32 columns: where
//   requests have fewer drafts than the longest, 2 costs up to 18% more (20 requests of up to 16,000 tokens, 1 to 5 drafts and 6
//   heads: 55 / 57, with 2 60 / 67); where all have as many, it is from 13% less (5 each: 71 / 75, with 2 62 / 70) to 8% more.
int col_tiles(int32_t G, int32_t max_q, int32_t D) {
    const int64_t cols = int64_t(G) * max_q;
    return cols <= (D == 256 ? 32 : 16) ? 1 : cols <= 32 || D > 64 ? 2 : 4;
}

// Resident workgroups of a launch.
int64_t most_groups(int D, int NT) {
    return int64_t(device_compute_units()) * (NT == 1 && D <= 128 ? 3 : NT * D <= 256 ? 2 : 1);
}

struct Workspace {
    size_t parts, bytes;           // the joins lie at 0
};
Workspace layout(int NT, int D, int64_t groups) {
    const size_t joins = align256(size_t(groups) * sizeof(Join));
    return {joins, joins + size_t(groups) * kWaves * 2 * size_t(part_floats(16 * NT, D)) * sizeof(float)};
}

template <int D, int NT, bool F16>
void launch(const AttendArgs& a, int64_t groups, hipStream_t stream) {
    const size_t lds = size_t(a.B + 1) * sizeof(int64_t);
    allow_dynamic_lds(kv_attend_kernel<D, NT, F16>, lds);
    hipLaunchKernelGGL((kv_attend_kernel<D, NT, F16>), dim3(uint32_t(groups)), dim3(kAttendNT), lds, stream, a);
    if (groups > 1) {
        const int64_t stretches = int64_t(a.B) * a.H * a.subs * ((a.max_q + a.Q - 1) / a.Q);
        const int split = stretches * kJoinSplit <= groups ? kJoinSplit : 1;
        hipLaunchKernelGGL((kv_join_kernel<D, NT, F16>), dim3(uint32_t(groups), uint32_t(split)), dim3(kJoinNT), 0, stream, a);
    }
}

template <int D, bool F16>
void launch(int NT, const AttendArgs& a, int64_t groups, hipStream_t stream) {
    if (NT == 1) launch<D, 1, F16>(a, groups, stream);
    else if (NT == 2) launch<D, 2, F16>(a, groups, stream);
    else if constexpr (D == 64) launch<D, 4, F16>(a, groups, stream);
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace
}  // namespace maps

using namespace maps;

extern "C" size_t maps_kv_attend_workspace_size(int32_t B, int64_t T, int32_t q_heads, int32_t heads, int32_t dim,
                                                int32_t max_q) {
    if (B < 1 || T < 1 || heads < 1 || q_heads < heads || q_heads % heads || !kv::dim_ok(dim) || max_q < 1) return 0;
    const int NT = col_tiles(q_heads / heads, max_q < T ? max_q : int32_t(T), dim);
    return layout(NT, dim, most_groups(dim, NT)).bytes;
}

extern "C" maps_status maps_kv_attend(const void* cache, int32_t num_blocks, int32_t block_size, int32_t heads,
                                      int32_t dim, const void* q, int32_t dtype, int64_t T, int32_t q_heads,
                                      int64_t q_stride_t, int64_t q_stride_h, const int32_t* table, int32_t B,
                                      int32_t max_blocks, const int32_t* lens, const int64_t* tok_off,
                                      int32_t max_q, float scale, int32_t window, void* out, float* lse,
                                      uint32_t* dev_err, void* workspace, size_t workspace_bytes,
                                      hipStream_t stream) {
    if (num_blocks < 1 || !kv::block_ok(block_size) || heads < 1 || !kv::dim_ok(dim) || T < 0 || T > INT32_MAX ||
        q_heads < 1 || q_heads % heads || B < 1 || B > MAPS_MAX_STEP_REQUESTS || max_blocks < 1 ||
        int64_t(B) * max_blocks > INT32_MAX || max_q < 1 || window < 0 || T * q_heads > INT32_MAX ||
        heads * kv::page_bytes(block_size, dim) > UINT32_MAX)
        return MAPS_E_SIZE;
    if (dtype != MAPS_BF16 && dtype != MAPS_F16) return MAPS_E_TYPE;
    if (!cache || !table || !lens || !tok_off || !dev_err || (T > 0 && (!q || !out))) return MAPS_E_NULL;
    if (!aligned(cache, 16) || !aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) ||
        (T > 1 && q_stride_t % 8) || (q_heads > 1 && q_stride_h % 8))   // (one row needs no stride)
        return MAPS_E_ALIGN;
    if (T == 0) return MAPS_OK;
    if (max_q > T) max_q = int32_t(T);
    const int32_t G = q_heads / heads;
    const int NT = col_tiles(G, max_q, dim);
    const int cols = 16 * NT, heads_per = G < cols ? G : cols, Q = cols / heads_per;
    const int subs = (G + heads_per - 1) / heads_per;
    // no more workgroups than the tables can hold stretches for
    const double tiles = double(max_blocks) * block_size / kTile + 1;
    const double all = double(B) * heads * subs * ((max_q + Q - 1) / Q) * (tiles + kSetUp) / (kMinTiles * kWaves) + 1;
    int64_t groups = most_groups(dim, NT);
    if (all < double(groups)) groups = int64_t(all);
    const Workspace ws = layout(NT, dim, groups);
    if (!workspace) return MAPS_E_NULL;
    if (workspace_bytes < ws.bytes) return MAPS_E_WORKSPACE;
    AttendArgs a{};
    a.cache = static_cast<const char*>(cache);
    a.num_blocks = num_blocks;
    a.shift = __builtin_ctz(unsigned(block_size));
    a.H = heads;
    a.Hq = q_heads;
    a.G = G;
    a.B = B;
    a.max_blocks = max_blocks;
    a.max_q = max_q;
    a.window = window;
    a.heads_per = heads_per;
    a.Q = Q;
    a.subs = subs;
    a.page = kv::page_bytes(block_size, dim);
    a.block = uint32_t(a.page * heads);
    a.v_skip = uint32_t(a.page / 2);
    a.T = T;
    a.q_st = q_stride_t;
    a.q_sh = q_stride_h;
    a.q = q;
    a.table = table;
    a.lens = lens;
    a.tok_off = tok_off;
    a.scale = scale;
    a.out = out;
    a.lse = lse;
    a.dev_err = dev_err;
    a.joins = static_cast<Join*>(workspace);
    a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + ws.parts);
    const bool f16 = dtype == MAPS_F16;
    if (dim == 64) f16 ? launch<64, true>(NT, a, groups, stream) : launch<64, false>(NT, a, groups, stream);
    else if (dim == 128) f16 ? launch<128, true>(NT, a, groups, stream) : launch<128, false>(NT, a, groups, stream);
    else f16 ? launch<256, true>(NT, a, groups, stream) : launch<256, false>(NT, a, groups, stream);
    MAPS_CHECK_LAUNCH();
    return MAPS_OK;
}
