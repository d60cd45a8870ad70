// Writing keys and values into the 4-bit cache and reading them back.
//
// A thread takes 8 consecutive channels of one token and head, of the key and
// of the value: 16 bytes in each as 16-bit numbers.  The four threads that
// share a scale are neighbours and exchange their largest magnitude by lane
// moves; the codes come from the conversion instruction, which rounds x / 2^e
// to the nearest E2M1 number, ties to the even code, and stops at 6.  Memory
// bound: values in and 17/32 bytes a value out.  32,768 tokens of 8 heads of 128
// channels: appended in 35 us from 16-bit types (4.9 TB/s) and in 57 from f32
// (5.3), read back in 31 (5.4) and 79 (3.9).
#include "kv_page.hpp"

namespace maps {
namespace {

constexpr int kRowNT = 256;

struct CacheArgs {
    char* cache;
    int32_t num_blocks, S, shift, H;      // shift: log2(S)
    int64_t page, T;
    const void *k, *v;                    // values of append
    void *k_out, *v_out;                  // values of read
    int64_t k_st, k_sh, v_st, v_sh;
    const int64_t* slots;
    uint32_t* dev_err;
};

template <int TYPE> struct Elem;
template <> struct Elem<MAPS_BF16> { using type = __bf16; };
template <> struct Elem<MAPS_F16> { using type = _Float16; };
template <> struct Elem<MAPS_F32> { using type = float; };

// 8 consecutive values as floats; whole 16-byte loads when the caller's arrays allow it.
template <int TYPE, bool VEC>
__device__ inline void load8(const typename Elem<TYPE>::type* p, float* x) {
    using T = typename Elem<TYPE>::type;
    if constexpr (VEC) {
        T e[8];
#pragma unroll
        for (int i = 0; i < int(sizeof(T)) / 2; ++i)
            reinterpret_cast<kv::u32x4*>(e)[i] = reinterpret_cast<const kv::u32x4*>(p)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = float(e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = float(p[i]);
    }
}

// The largest of four neighbouring lanes' values.
__device__ inline uint32_t quad_max(uint32_t x) {
    const uint32_t y = uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0xB1, 0xf, 0xf, false));   // lanes 1 0 3 2
    x = x > y ? x : y;
    const uint32_t z = uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0x4E, 0xf, 0xf, false));   // lanes 2 3 0 1
    return x > z ? x : z;
}

// Codes of 8 values, and the scale byte that they share with their neighbours' 24.
__device__ inline uint32_t quantise(const float* x, uint32_t* byte) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;    // magnitudes order as their bits, NaN above all
        m = a > m ? a : m;
    }
    const uint32_t field = quad_max(m) >> 23;
    const uint32_t s = field < 2 + kv::kScaleMin ? kv::kScaleMin : field - 2;
    const float scale = kv::scale_value(s);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
    *byte = field == 255 ? kv::kScaleNan : s;
    return field == 255 ? 0 : c;
}

template <int D, int TYPE, bool VEC>
__global__ __launch_bounds__(kRowNT) void kv_append_kernel(CacheArgs a) {
    using T = typename Elem<TYPE>::type;
    constexpr int P = D / 8;                              // threads a token and head
    const int64_t rows = a.T * a.H;
    const int part = threadIdx.x % P;
    for (int64_t row = int64_t(blockIdx.x) * (kRowNT / P) + threadIdx.x / P; row < rows;
         row += int64_t(gridDim.x) * (kRowNT / P)) {
        const int64_t t = row / a.H;
        const int h = int(row - t * a.H);
        const int64_t slot = a.slots[t];
        if (slot < 0) continue;                           // (whole groups of P threads leave together)
        if ((slot >> a.shift) >= a.num_blocks) {
            if (part == 0 && h == 0) raise_error(a.dev_err, MAPS_ERR_SLOT);
            continue;
        }
        const int at = int(slot & (a.S - 1));
        char* page = a.cache + ((slot >> a.shift) * a.H + h) * a.page;
        float x[8], y[8];
        load8<TYPE, VEC>(static_cast<const T*>(a.k) + t * a.k_st + h * a.k_sh + part * 8, x);
        load8<TYPE, VEC>(static_cast<const T*>(a.v) + t * a.v_st + h * a.v_sh + part * 8, y);
        uint32_t ks, vs;
        const uint32_t kc = quantise(x, &ks), vc = quantise(y, &vs);
        *reinterpret_cast<uint32_t*>(page + at * (D / 2) + part * 4) = kc;
        char* k_scales = page + kv::codes_bytes(a.S, D);
        char* v_codes = k_scales + kv::scales_bytes(a.S, D);
        char* v_scales = v_codes + kv::codes_bytes(a.S, D);
        if (part % 4 == 0) {
            k_scales[at * (D / 32) + part / 4] = char(ks);
            v_scales[kv::v_scale(at, part / 4, D)] = char(vs);
        }
        if constexpr (D == 64) {                          // two channel groups of 4
            *reinterpret_cast<uint16_t*>(v_codes + kv::v_code(at, 2 * part, 0, D)) = uint16_t(vc);
            *reinterpret_cast<uint16_t*>(v_codes + kv::v_code(at, 2 * part + 1, 0, D)) = uint16_t(vc >> 16);
        } else {                                          // one group of 8, or half of one of 16
            constexpr int Q = D / 128;
            *reinterpret_cast<uint32_t*>(v_codes + kv::v_code(at, part / Q, part % Q * 4, D)) = vc;
        }
    }
}

template <int TYPE>
__device__ inline void store8(typename Elem<TYPE>::type* p, uint32_t codes, uint32_t byte) {
    using T = typename Elem<TYPE>::type;
    const float scale = kv::scale_value(byte);
    const kv::f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3)};
    T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = T(v[i / 2][i % 2]);
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; ++i)
        reinterpret_cast<kv::u32x4*>(p)[i] = reinterpret_cast<kv::u32x4*>(e)[i];
}

template <int D, int TYPE>
__global__ __launch_bounds__(kRowNT) void kv_read_kernel(CacheArgs a) {
    using T = typename Elem<TYPE>::type;
    constexpr int P = D / 8;
    const int64_t rows = a.T * a.H;
    const int part = threadIdx.x % P;
    for (int64_t row = int64_t(blockIdx.x) * (kRowNT / P) + threadIdx.x / P; row < rows;
         row += int64_t(gridDim.x) * (kRowNT / P)) {
        const int64_t t = row / a.H;
        const int h = int(row - t * a.H);
        const int64_t slot = a.slots[t];
        uint32_t kc = 0, vc = 0, ks = kv::kScaleOne, vs = kv::kScaleOne;
        if (slot >= 0 && (slot >> a.shift) < a.num_blocks) {
            const int at = int(slot & (a.S - 1));
            const char* page = a.cache + ((slot >> a.shift) * a.H + h) * a.page;
            const char* k_scales = page + kv::codes_bytes(a.S, D);
            const char* v_codes = k_scales + kv::scales_bytes(a.S, D);
            const char* v_scales = v_codes + kv::codes_bytes(a.S, D);
            kc = *reinterpret_cast<const uint32_t*>(page + at * (D / 2) + part * 4);
            ks = uint8_t(k_scales[at * (D / 32) + part / 4]);
            vs = uint8_t(v_scales[kv::v_scale(at, part / 4, D)]);
            if constexpr (D == 64) {
                vc = *reinterpret_cast<const uint16_t*>(v_codes + kv::v_code(at, 2 * part, 0, D)) |
                     uint32_t(*reinterpret_cast<const uint16_t*>(v_codes + kv::v_code(at, 2 * part + 1, 0, D))) << 16;
            } else {
                constexpr int Q = D / 128;
                vc = *reinterpret_cast<const uint32_t*>(v_codes + kv::v_code(at, part / Q, part % Q * 4, D));
            }
        } else if (slot >= 0 && part == 0 && h == 0) {
            raise_error(a.dev_err, MAPS_ERR_SLOT);
        }
        store8<TYPE>(static_cast<T*>(a.k_out) + row * D + part * 8, kc, ks);
        store8<TYPE>(static_cast<T*>(a.v_out) + row * D + part * 8, vc, vs);
    }
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

maps_status check(const void* cache, int32_t num_blocks, int32_t S, int32_t H, int32_t D, int32_t dtype, int64_t T) {
    if (num_blocks < 1 || !kv::block_ok(S) || H < 1 || !kv::dim_ok(D) || T < 0 || T > INT32_MAX) return MAPS_E_SIZE;
    if (dtype != MAPS_BF16 && dtype != MAPS_F16 && dtype != MAPS_F32) return MAPS_E_TYPE;
    if (!cache) return MAPS_E_NULL;
    return aligned(cache, 16) ? MAPS_OK : MAPS_E_ALIGN;
}

CacheArgs args(const void* cache, int32_t num_blocks, int32_t S, int32_t H, int32_t D, int64_t T,
               const int64_t* slots, uint32_t* dev_err) {
    CacheArgs a{};
    a.cache = static_cast<char*>(const_cast<void*>(cache));
    a.num_blocks = num_blocks;
    a.S = S;
    a.shift = __builtin_ctz(unsigned(S));
    a.H = H;
    a.page = kv::page_bytes(S, D);
    a.T = T;
    a.slots = slots;
    a.dev_err = dev_err;
    return a;
}

template <typename F>
maps_status for_dim(int32_t D, F f) {
    if (D == 64) f(std::integral_constant<int, 64>{});
    else if (D == 128) f(std::integral_constant<int, 128>{});
    else f(std::integral_constant<int, 256>{});
    MAPS_CHECK_LAUNCH();
    return MAPS_OK;
}

template <typename F>
maps_status for_type(int32_t D, int32_t dtype, F f) {
    return for_dim(D, [&](auto d) {
        if (dtype == MAPS_BF16) f(d, std::integral_constant<int, MAPS_BF16>{});
        else if (dtype == MAPS_F16) f(d, std::integral_constant<int, MAPS_F16>{});
        else f(d, std::integral_constant<int, MAPS_F32>{});
    });
}

dim3 row_grid(int64_t T, int32_t H, int32_t D) {
    const int64_t wgs = (T * H * (D / 8) + kRowNT - 1) / kRowNT, most = int64_t(device_compute_units()) * 32;
    return dim3(uint32_t(wgs < most ? wgs : most));
}

}  // namespace
}  // namespace maps

using namespace maps;

extern "C" size_t maps_kv_page_bytes(int32_t block_size, int32_t dim) {
    return kv::block_ok(block_size) && kv::dim_ok(dim) ? size_t(kv::page_bytes(block_size, dim)) : 0;
}

extern "C" maps_status maps_kv_append(void* cache, int32_t num_blocks, int32_t block_size, int32_t heads, int32_t dim,
                                      const void* k, const void* v, int32_t dtype, int64_t T, int64_t k_stride_t,
                                      int64_t k_stride_h, int64_t v_stride_t, int64_t v_stride_h,
                                      const int64_t* slots, uint32_t* dev_err, hipStream_t stream) {
    const maps_status st = check(cache, num_blocks, block_size, heads, dim, dtype, T);
    if (st != MAPS_OK) return st;
    if (!dev_err || (T > 0 && (!k || !v || !slots))) return MAPS_E_NULL;
    const int bytes = kv::type_bytes(dtype);
    if (!aligned(k, bytes) || !aligned(v, bytes)) return MAPS_E_ALIGN;
    if (T == 0) return MAPS_OK;
    CacheArgs a = args(cache, num_blocks, block_size, heads, dim, T, slots, dev_err);
    a.k = k;
    a.v = v;
    a.k_st = k_stride_t;
    a.k_sh = k_stride_h;
    a.v_st = v_stride_t;
    a.v_sh = v_stride_h;
    // 16-byte loads where every row of 8 channels starts on a 16-byte boundary
    const int per = 16 / bytes;
    const bool vec = aligned(k, 16) && aligned(v, 16) &&
                     (k_stride_t % per | k_stride_h % per | v_stride_t % per | v_stride_h % per) == 0;
    const dim3 grid = row_grid(T, heads, dim);
    return for_type(dim, dtype, [&](auto d, auto ty) {
        if (vec)
            hipLaunchKernelGGL((kv_append_kernel<d(), ty(), true>), grid, dim3(kRowNT), 0, stream, a);
        else
            hipLaunchKernelGGL((kv_append_kernel<d(), ty(), false>), grid, dim3(kRowNT), 0, stream, a);
    });
}

extern "C" maps_status maps_kv_read(const void* cache, int32_t num_blocks, int32_t block_size, int32_t heads,
                                    int32_t dim, const int64_t* slots, int64_t T, void* k_out, void* v_out,
                                    int32_t dtype, uint32_t* dev_err, hipStream_t stream) {
    const maps_status st = check(cache, num_blocks, block_size, heads, dim, dtype, T);
    if (st != MAPS_OK) return st;
    if (!dev_err || (T > 0 && (!slots || !k_out || !v_out))) return MAPS_E_NULL;
    if (!aligned(k_out, 16) || !aligned(v_out, 16)) return MAPS_E_ALIGN;
    if (T == 0) return MAPS_OK;
    CacheArgs a = args(cache, num_blocks, block_size, heads, dim, T, slots, dev_err);
    a.k_out = k_out;
    a.v_out = v_out;
    const dim3 grid = row_grid(T, heads, dim);
    return for_type(dim, dtype, [&](auto d, auto ty) {
        hipLaunchKernelGGL((kv_read_kernel<d(), ty()>), grid, dim3(kRowNT), 0, stream, a);
    });
}
