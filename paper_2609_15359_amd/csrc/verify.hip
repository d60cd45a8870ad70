// Verification of drafted tokens against the target's probabilities.
//
// The accepted drafts of a request take K gathers; the next token is an
// exponential race over the vocabulary, max_i w_i / e_i.  A maximum depends on
// no order, so a row is cut into pieces of one workgroup each, every piece
// keeps its best entry as one 64-bit key (the score's bits above the
// complemented index: the lowest index wins ties), and a second launch takes
// the best piece.  A request's K comparisons are repeated by each of its
// pieces.  Memory bound: one row of the target, one of the noise and, after a
// refusal, one of the drafts.  256 requests with 4 drafts over 131,072 entries,
// 179 of them refused: 76 us in f32 = 4.8 TB/s (single entries a load: 96; 8
// entries a thread: 127; the noise loaded ahead of the drafts' comparison: 162,
// its registers leave half of the wavefronts), 54 in 16-bit types = 4.6.
#include "kv_page.hpp"

namespace maps {
namespace {

constexpr int kVerifyNT = 256;
constexpr int kPiece = 8192;          // entries of a row that one workgroup takes

struct VerifyArgs {
    int32_t B, K, V, pieces;
    const void *target, *draft;
    int64_t t_b, t_j, d_b, d_j;
    const int32_t *draft_tokens, *n_draft;
    const float *u, *noise;
    int64_t noise_stride;
    int32_t *tokens, *accepted;
    uint32_t* dev_err;
    uint64_t* best;                   // [B][pieces][2]: of w, and of p alone
};

template <int TYPE> struct Prob;
template <> struct Prob<MAPS_BF16> { using type = __bf16; };
template <> struct Prob<MAPS_F16> { using type = _Float16; };
template <> struct Prob<MAPS_F32> { using type = float; };

// The number of accepted drafts of request b; every lane of the wavefront gets it.
template <int TYPE>
__device__ inline int accepted_drafts(const VerifyArgs& a, int b, int n, uint32_t* err) {
    using T = typename Prob<TYPE>::type;
    const int j = threadIdx.x % kWave;
    bool take = false;
    if (j < n) {
        const int32_t x = a.draft_tokens[int64_t(b) * a.K + j];
        if (uint32_t(x) >= uint32_t(a.V)) {
            *err |= MAPS_ERR_DRAFT;
        } else {
            const float p = float(static_cast<const T*>(a.target)[b * a.t_b + j * a.t_j + x]);
            const float q = a.draft ? float(static_cast<const T*>(a.draft)[b * a.d_b + j * a.d_j + x]) : 1.0f;
            take = a.u[int64_t(b) * a.K + j] * q < p;
        }
    }
    const uint64_t stops = ~__ballot(take) | (n < kWave ? 1ull << n : 0ull);
    return stops ? __builtin_ctzll(stops) : kWave;
}

__device__ inline int draft_count(const VerifyArgs& a, int b, uint32_t* err) {
    const int n = a.n_draft[b];
    if (n < -1 || n > a.K) *err |= MAPS_ERR_DRAFT;
    return n < -1 ? -1 : n > a.K ? a.K : n;
}

__device__ inline uint64_t race_key(float w, float noise, int i) {
    const float score = w / noise;
    return w > 0.0f && score >= 0.0f ? (uint64_t(__float_as_uint(score)) << 32) | ~uint32_t(i) : 0;
}

__device__ inline uint64_t best_of(uint64_t x, uint64_t y) { return x > y ? x : y; }

// Entries i .. i + 3 of a row as floats, 0 from `end` on.  A row may start anywhere: the load asks for no more than its
// type's alignment, which this chip's wide global loads do not need.
template <typename T>
__device__ inline void load4(const T* row, uint32_t i, uint32_t end, float* x) {
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (i + 4 <= end) {
        const vec y = *reinterpret_cast<const vec*>(row + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = float(y[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = i + k < end ? float(row[i + k]) : 0.0f;
    }
}

template <int TYPE>
__global__ __launch_bounds__(kVerifyNT) void race_kernel(VerifyArgs a) {
    using T = typename Prob<TYPE>::type;
    const int b = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces;
    const uint32_t from = uint32_t(piece) * kPiece;         // (rows of nearly 2^31 entries: sums below stay inside 32 bits)
    const uint32_t end = uint32_t(a.V) - from < kPiece ? uint32_t(a.V) : from + kPiece;
    // (the noise is the same row whatever is accepted, but loading it ahead of the comparisons costs wavefronts)
    const float* noise = a.noise + b * a.noise_stride;
    constexpr int kRounds = kPiece / (4 * kVerifyNT);
    uint32_t err = 0;
    const int n = draft_count(a, b, &err);
    if (n < 0) return;
    const int acc = n > 0 ? accepted_drafts<TYPE>(a, b, n, &err) : 0;
    const bool refused = acc < n;
    const T* p = static_cast<const T*>(a.target) + b * a.t_b + acc * a.t_j;
    const T* q = refused && a.draft ? static_cast<const T*>(a.draft) + b * a.d_b + acc * a.d_j : nullptr;
    const int only = refused && !a.draft ? a.draft_tokens[int64_t(b) * a.K + acc] : -1;
    uint64_t best = 0, plain = 0;
#pragma unroll 2
    for (int r = 0; r < kRounds; ++r) {
        const uint32_t i0 = from + (r * kVerifyNT + threadIdx.x) * 4;
        float pi[4], qi[4] = {}, e[4];
        load4(noise, i0, end, e);
        load4(p, i0, end, pi);
        if (q) load4(q, i0, end, qi);
#pragma unroll
        for (int i = 0; i < 4; ++i) {                      // (entries past the row are 0 and never win)
            const float w = int(i0 + i) == only ? 0.0f : pi[i] - qi[i];
            best = best_of(best, race_key(w, e[i], int(i0) + i));
            if (refused) plain = best_of(plain, race_key(pi[i], e[i], int(i0) + i));
        }
    }
    __shared__ uint64_t tmp[kVerifyNT / kWave];
    best = block_reduce_max<kVerifyNT>(best, tmp);
    __syncthreads();
    if (refused) plain = block_reduce_max<kVerifyNT>(plain, tmp);
    if (threadIdx.x == 0) {
        a.best[int64_t(blockIdx.x) * 2] = best;
        a.best[int64_t(blockIdx.x) * 2 + 1] = plain;
    }
}

template <int TYPE>
__global__ __launch_bounds__(kWave) void verify_kernel(VerifyArgs a) {
    const int b = blockIdx.x, lane = threadIdx.x;
    uint32_t err = 0;
    const int n = draft_count(a, b, &err);
    const int acc = n > 0 ? accepted_drafts<TYPE>(a, b, n, &err) : 0;
    int32_t next = -1;
    if (n >= 0) {
        uint64_t best = 0, plain = 0;
        for (int i = lane; i < a.pieces; i += kWave) {
            best = best_of(best, a.best[(int64_t(b) * a.pieces + i) * 2]);
            plain = best_of(plain, a.best[(int64_t(b) * a.pieces + i) * 2 + 1]);
        }
        best = wave_reduce_max(best);
        plain = wave_reduce_max(plain);
        if (!best) best = plain;
        if (best) next = int32_t(~uint32_t(best));
        else err |= MAPS_ERR_DRAFT;
    }
    for (int j = lane; j <= a.K; j += kWave)
        a.tokens[int64_t(b) * (a.K + 1) + j] =
            n < 0 || j > acc ? -1 : j == acc ? next : a.draft_tokens[int64_t(b) * a.K + j];
    if (lane == 0) a.accepted[b] = n < 0 ? -1 : acc;
    if (err) raise_error(a.dev_err, err);
}

int32_t pieces_of(int32_t V) { return (V - 1) / kPiece + 1; }

template <int TYPE>
void launch(const VerifyArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((race_kernel<TYPE>), dim3(uint32_t(a.B) * uint32_t(a.pieces)), dim3(kVerifyNT), 0, stream, a);
    hipLaunchKernelGGL((verify_kernel<TYPE>), dim3(uint32_t(a.B)), dim3(kWave), 0, stream, a);
}

}  // namespace
}  // namespace maps

using namespace maps;

extern "C" size_t maps_verify_drafts_workspace_size(int32_t B, int32_t V) {
    return B < 1 || V < 1 ? 0 : size_t(B) * size_t(pieces_of(V)) * 2 * sizeof(uint64_t);
}

extern "C" maps_status maps_verify_drafts(int32_t B, int32_t K, int32_t V, const void* target,
                                          int64_t target_stride_b, int64_t target_stride_j, const void* draft,
                                          int64_t draft_stride_b, int64_t draft_stride_j, int32_t dtype,
                                          const int32_t* draft_tokens, const int32_t* n_draft, const float* u,
                                          const float* noise, int64_t noise_stride, int32_t* tokens,
                                          int32_t* accepted, uint32_t* dev_err, void* workspace,
                                          size_t workspace_bytes, hipStream_t stream) {
    if (B < 1 || K < 0 || K > MAPS_MAX_DRAFTS || V < 1) return MAPS_E_SIZE;
    if (int64_t(B) * pieces_of(V) > INT32_MAX) return MAPS_E_SIZE;
    if (dtype != MAPS_BF16 && dtype != MAPS_F16 && dtype != MAPS_F32) return MAPS_E_TYPE;
    if (!target || !n_draft || !noise || !tokens || !accepted || !dev_err || !workspace ||
        (K > 0 && (!draft_tokens || !u)))
        return MAPS_E_NULL;
    if (reinterpret_cast<uintptr_t>(workspace) % 8) return MAPS_E_ALIGN;
    if (workspace_bytes < maps_verify_drafts_workspace_size(B, V)) return MAPS_E_WORKSPACE;
    VerifyArgs a{};
    a.B = B;
    a.K = K;
    a.V = V;
    a.pieces = pieces_of(V);
    a.target = target;
    a.draft = draft;
    a.t_b = target_stride_b;
    a.t_j = target_stride_j;
    a.d_b = draft_stride_b;
    a.d_j = draft_stride_j;
    a.draft_tokens = draft_tokens;
    a.n_draft = n_draft;
    a.u = u;
    a.noise = noise;
    a.noise_stride = noise_stride;
    a.tokens = tokens;
    a.accepted = accepted;
    a.dev_err = dev_err;
    a.best = static_cast<uint64_t*>(workspace);
    if (dtype == MAPS_BF16) launch<MAPS_BF16>(a, stream);
    else if (dtype == MAPS_F16) launch<MAPS_F16>(a, stream);
    else launch<MAPS_F32>(a, stream);
    MAPS_CHECK_LAUNCH();
    return MAPS_OK;
}
