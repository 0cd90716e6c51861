// matvec.hip - dense products of a few rows with 4-bit weights: y[t] = W x[t], the
// weights e2m1 numbers with a power-of-two scale for every 32 of a row (mx4.h).
//
// The weights are all there is to read, each used for a handful of products, so the
// kernels are streams of them.  A tile is 16 weight rows by up to 16 rows of x: lane (r, q)
// = 16 q + r has 16 bytes, a block of 32 values, of weight row r, makes bf16 of them, scale
// and all, and the bf16 matrix core multiplies; an fp32 x is the sum of three bf16
// numbers, exactly but for what lies below 2^-133, the smallest of them.
#include <algorithm>

#include "product.h"

namespace cmoe {

namespace {

constexpr int kLine = 256;  // values of 128 bytes of weights

// The first part of a finite number is cut off, not rounded: of the largest ones the nearest
// bf16 number would be infinity.  What is left has 16 bits, and the second part's rest 8.
__device__ inline void split3(float v, __bf16* p) {
    const bool finite = fabsf(v) < INFINITY;
    const float top = finite ? __uint_as_float(__float_as_uint(v) & 0xFFFF0000u) : v, r = finite ? v - top : 0.0f;
    p[0] = (__bf16)top;
    p[1] = (__bf16)r;
    p[2] = (__bf16)(r - (float)p[1]);
}

// Rows of x of the launch, which begin at row0 of the call's.
__device__ inline int live_rows(const MatvecArgs& a) { return a.n_rows ? min(max(*a.n_rows, 0) - a.row0, a.rows) : a.rows; }

// Products of a block of 32 weights with the same values of x, eight at a time.
template <int PLANES>
__device__ __forceinline__ f32x4 multiply(const u32x4& w, uint32_t byte, const u32x4 (&x)[PLANES][4], f32x4 c) {
    const float s = mx_scale(byte);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bf16x8 wide = __builtin_bit_cast(bf16x8, widen4(w[j], s));
#pragma unroll
        for (int p = PLANES - 1; p >= 0; --p) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide, __builtin_bit_cast(bf16x8, x[p][j]), c, 0, 0, 0);
    }
    return c;
}

// fp32 rows, whose products are added up three times as often and to more bits: a line of
// 256 values is a chain of its own.  y off by, rms, for 4096 values 1.6e-7 in the wide kernel,
// in one chain 5.5e-7; for 65536, 3.4e-7 and 2.1e-6, in the narrow one 1.9e-7 and 5.7e-7.  At
// 131072 x 4096, 1 and 21 fp32 rows, 55.0 and 134 us, without 53.7 and 132; 2880 x 4096, 16
// rows, 13.1 both.
__device__ __forceinline__ void end_chain(f32x4& sum, f32x4& chain) {
    sum += chain;
    chain = f32x4{};
}

// Columns j .. j + 3 of row t of y.
__device__ __forceinline__ void put(const MatvecArgs& a, int64_t t, int64_t j, const f32x4& v) {
    const int64_t at = t * a.y_stride + j;
    if (a.y_bf16) {
        __bf16* y = static_cast<__bf16*>(a.y) + at;
        if (a.y_aligned && j + 3 < a.m)
            *reinterpret_cast<bf16x4*>(y) = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
        else
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (j + k < a.m) y[k] = (__bf16)v[k];
    } else {
        float* y = static_cast<float*>(a.y) + at;
        if (a.y_aligned && j + 3 < a.m)
            *reinterpret_cast<f32x4*>(y) = v;
        else
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (j + k < a.m) y[k] = v[k];
    }
}

// ---------------------------------------------------------------- few weight rows
// A workgroup takes a tile, its wavefronts share the row's lines of 128 bytes, and
// everything goes straight into the matrix core's registers: there is no wait but the
// one for memory, and the sum over the wavefronts.  4096 x 2048, one bf16 row, 4.4 us, a
// launch and one trip to memory; 2880 x 4096, sixteen fp32 rows, 14.5 (with 8 wavefronts
// and two lines of registers 15.0): each wavefront splits the same rows of x again.
// grid: x = tiles, y = rows of x / 16, rounded up
constexpr int kNarrowWaves = 16;  // at most
template <bool BF16>
__global__ __launch_bounds__(64 * kNarrowWaves) void matvec_narrow_kernel(MatvecArgs a) {
    constexpr int PLANES = BF16 ? 1 : 3, kUnits = BF16 ? 4 : 8;  // 16-byte units of a block of x
    __shared__ f32x4 red[kNarrowWaves][64];
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, waves = blockDim.x >> 6;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t0 = blockIdx.y * 16, n = min(live_rows(a) - t0, 16);
    if (n <= 0) return;
    const int blocks = a.d / 32, lines = (blocks + 7) / 8;
    const int64_t row = std::min<int64_t>((int64_t)blockIdx.x * 16 + r, a.m - 1);
    const uint8_t *w = a.w + row * a.w_pitch, *scale = a.w_scale + row * a.w_scale_pitch;
    const char* x = static_cast<const char*>(a.x) + (t0 + min(r, n - 1)) * a.x_stride * (BF16 ? 2 : 4);
    struct Line {
        u32x4 w[2], x[2][kUnits];
        uint32_t scale[2];
    };
    auto load = [&](int l, Line& v) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int b = l * 8 + 4 * h + q;
            const bool in = b < blocks;  // zeros behind the row's end
            v.w[h] = in ? *reinterpret_cast<const u32x4*>(w + (int64_t)b * 16) : u32x4{};
            v.scale[h] = in ? scale[b] : 0;
#pragma unroll
            for (int u = 0; u < kUnits; ++u) v.x[h][u] = in && r < n ? *reinterpret_cast<const u32x4*>(x + ((int64_t)b * kUnits + u) * 16) : u32x4{};
        }
    };
    f32x4 acc = {};
    auto step = [&](const Line& v) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 p[PLANES][4];
            if constexpr (BF16) {
#pragma unroll
                for (int j = 0; j < 4; ++j) p[0][j] = v.x[h][j];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    bf16x8 b[3];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        __bf16 s[3];
                        split3(__uint_as_float(v.x[h][2 * j + k / 4][k % 4]), s);
                        b[0][k] = s[0];
                        b[1][k] = s[1];
                        b[2][k] = s[2];
                    }
#pragma unroll
                    for (int k = 0; k < 3; ++k) p[k][j] = __builtin_bit_cast(u32x4, b[k]);
                }
            }
            acc = multiply<PLANES>(v.w[h], v.scale[h], p, acc);
        }
    };
    if constexpr (BF16) {
        Line v, next;
        int l = wv;
        if (l < lines) load(l, v);
        for (; l < lines; l += waves) {
            if (l + waves < lines) load(l + waves, next);
            step(v);
            v = next;
        }
    } else {  // registers for one line of fp32 values
        f32x4 sum = {};
        for (int l = wv; l < lines; l += waves) {
            Line v;
            load(l, v);
            step(v);
            end_chain(sum, acc);
        }
        acc = sum;
    }
    red[wv][lane] = acc;
    __syncthreads();
    if (wv) return;
    for (int k = 1; k < waves; ++k) acc += red[k][lane];
    if (r < n) put(a, t0 + r, (int64_t)blockIdx.x * 16 + 4 * q, acc);
}

// ---------------------------------------------------------------- many weight rows
// Weights come as lines of 128 bytes, eight rows an instruction, and through a
// wavefront's part of LDS into the matrix core's order (units q and q + 4 of row r for
// lane (r, q)); loaded straight into registers they would come sixteen lines an
// instruction, half of each.  x lies in LDS for the whole workgroup, `chunk` lines of it
// at a time, and its next chunk is on the way in registers meanwhile.
// Bound by HBM: 131072 x 4096, one row of x, 47.3 us, 6.0 TB/s.  Rows that are no whole
// lines of memory, 131075 x 2880, five rows, 44.2 us, 4.6 TB/s: a load of 128 bytes takes
// parts of two lines there.  With 64 rows of x by x's reads from LDS: 131072 x 4096 in
// 130 us.  A line of more than 21 fp32 rows does not fit into x's LDS, so they are launches
// of 21, which read the weights each: 22 and 64 rows, 131072 x 4096, in 192 and 459 us.
// G: groups of 16 rows of x.  WHOLE: rows of whole lines of memory, which are read once,
// nontemporally; elsewhere the caches keep a line's other part (46 us against 53.5).
// fp32 rows: registers for four wavefronts a SIMD, two workgroups a CU; left to itself the
// compiler takes 139 for two tiles, and 131072 x 4096 takes 56.2 us instead of 55.0.
// grid: x = tiles / (RT kWaves) rounded up
constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kXBytes = 32 * 1024;  // of LDS for x

template <int PLANES, int RT, int G, bool WHOLE>
__global__ __launch_bounds__(kThreads, PLANES == 3 ? 4 : 1) void matvec_wide_kernel(MatvecArgs a, int columns, int chunk) {
    constexpr int kMine = (kXBytes / (PLANES * 16) + kThreads - 1) / kThreads;  // blocks of eight values of a chunk, per thread
    __shared__ __align__(16) char xs[kXBytes];
    __shared__ __align__(16) char ws[kWaves][RT * 2048];
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, q = lane >> 4, i8 = lane >> 3, p8 = lane & 7;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = min(columns, live_rows(a));
    if (n <= 0) return;
    const int tile0 = (blockIdx.x * kWaves + wv) * RT, all = (a.m + 15) / 16;
    const int blocks = a.d / 32, lines = (blocks + 7) / 8;

    const uint8_t *w[RT][2], *scale[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int64_t row = (int64_t)(tile0 + t) * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) w[t][h] = a.w + std::min<int64_t>(row + 8 * h + i8, a.m - 1) * a.w_pitch;
        scale[t] = a.w_scale + std::min<int64_t>(row + (lane >> 2), a.m - 1) * a.w_scale_pitch;
    }
    auto load = [&](int l, u32x4 (&v)[RT][2]) {
        const int u = l * 8 + p8;
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                v[t][h] = u >= blocks ? u32x4{}
                          : WHOLE     ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(w[t][h] + (int64_t)u * 16))
                                      : *reinterpret_cast<const u32x4*>(w[t][h] + (int64_t)u * 16);
    };
    // scales of four lines from l: lane 4 i + c those of row i, line l + c
    auto load_scales = [&](int l, u32x2 (&s)[RT]) {
        const int at = (l + (lane & 3)) * 8;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            uint64_t v = 0;
            if (at + 8 <= blocks) {
                __builtin_memcpy(&v, scale[t] + at, 8);
            } else {
                for (int b = 0; b < 8; ++b)
                    if (at + b < blocks) v |= (uint64_t)scale[t][at + b] << (8 * b);
            }
            s[t] = __builtin_bit_cast(u32x2, v);
        }
    };
    // eight values of x per thread and step, zeros behind the row's end: block i of the
    // chunk from line c0
    auto load_x = [&](int c0, u32x4 (&e)[kMine][PLANES == 1 ? 1 : 2]) {
        const int blocks8 = (min(c0 + chunk, lines) - c0) * n * 32;
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int i = k * kThreads + tid, u = i & 31, c = (i >> 5) % n, l = (i >> 5) / n, at = (c0 + l) * kLine + u * 8;
            const bool in = i < blocks8 && at < a.d;
#pragma unroll
            for (int p = 0; p < (PLANES == 1 ? 1 : 2); ++p)
                e[k][p] = in ? *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.x) + ((a.row0 + c) * a.x_stride + at) * (PLANES == 1 ? 2 : 4) + p * 16)
                             : u32x4{};
        }
    };
    auto store_x = [&](int c0, const u32x4 (&e)[kMine][PLANES == 1 ? 1 : 2]) {
        const int blocks8 = (min(c0 + chunk, lines) - c0) * n * 32;
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int i = k * kThreads + tid, u = i & 31, c = (i >> 5) % n, l = (i >> 5) / n;
            if (i >= blocks8) break;
            char* to = xs + ((l * columns + c) * PLANES * 32 + (u ^ (c & 7))) * 16;
            if constexpr (PLANES == 1) {
                *reinterpret_cast<u32x4*>(to) = e[k][0];
            } else {
                bf16x8 p[3];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    __bf16 b[3];
                    split3(__uint_as_float(e[k][PLANES == 1 ? 0 : j / 4][j % 4]), b);
                    p[0][j] = b[0];
                    p[1][j] = b[1];
                    p[2][j] = b[2];
                }
#pragma unroll
                for (int j = 0; j < 3; ++j) *reinterpret_cast<bf16x8*>(to + j * 512) = p[j];
            }
        }
    };

    u32x4 v[RT][2], e[kMine][PLANES == 1 ? 1 : 2];
    u32x2 s[RT];
    load_x(0, e);
    if (tile0 < all) {
        load(0, v);
        load_scales(0, s);
    }
    f32x4 acc[RT][G] = {}, sum[RT][G] = {};
    char* const lds = ws[wv];
    for (int c0 = 0; c0 < lines; c0 += chunk) {
        const int c1 = min(c0 + chunk, lines);
        if (c0) __syncthreads();
        store_x(c0, e);
        __syncthreads();
        if (c1 < lines) load_x(c1, e);
        if (tile0 >= all) continue;
        for (int l = c0; l < c1; ++l) {
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) *reinterpret_cast<u32x4*>(lds + t * 2048 + h * 1024 + i8 * 128 + (p8 ^ i8) * 16) = v[t][h];
            uint32_t mine[RT][2];
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) mine[t][h] = (uint32_t)__shfl((int)s[t][h], 4 * r + (l & 3));
            if (l + 1 < lines) {
                load(l + 1, v);
                if ((l & 3) == 3) load_scales(l + 1, s);
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 u[RT];
                float f[RT];
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    u[t] = *reinterpret_cast<const u32x4*>(lds + t * 2048 + r * 128 + (((q + 4 * h) ^ (r & 7)) << 4));
                    f[t] = mx_scale((mine[t][h] >> (8 * q)) & 255u);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    bf16x8 wide[RT];
#pragma unroll
                    for (int t = 0; t < RT; ++t) wide[t] = __builtin_bit_cast(bf16x8, widen4(u[t][j], f[t]));
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const int c = min(16 * g + r, n - 1);  // columns past the last repeat it, and are dropped
                        const char* xl = xs + ((l - c0) * columns + c) * PLANES * 512 + ((((q + 4 * h) * 4 + j) ^ (c & 7)) << 4);
#pragma unroll
                        for (int p = PLANES - 1; p >= 0; --p) {
                            const bf16x8 b = *reinterpret_cast<const bf16x8*>(xl + p * 512);
#pragma unroll
                            for (int t = 0; t < RT; ++t) acc[t][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[t], b, acc[t][g], 0, 0, 0);
                        }
                    }
                }
            }
            if constexpr (PLANES == 3)
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int g = 0; g < G; ++g) end_chain(sum[t][g], acc[t][g]);
            __builtin_amdgcn_wave_barrier();
        }
    }
    if (tile0 >= all) return;
    // lane (r, q) holds rows 4 q .. of a tile for column r of a group
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (16 * g + r < n) put(a, a.row0 + 16 * g + r, (int64_t)(tile0 + t) * 16 + 4 * q, PLANES == 3 ? sum[t][g] : acc[t][g]);
}

template <int PLANES, int RT, int G>
void launch_wide(const MatvecArgs& a, hipStream_t st) {
    const bool whole = a.w_pitch % 128 == 0 && ((uintptr_t)a.w & 127) == 0;
    const int lines = (a.d + kLine - 1) / kLine, columns = a.rows, chunk = std::min(lines, kXBytes / (columns * PLANES * 512));
    const int64_t tiles = (a.m + 15) / 16;
    launch_kernel(whole ? matvec_wide_kernel<PLANES, RT, G, true> : matvec_wide_kernel<PLANES, RT, G, false>,
                  dim3((unsigned)((tiles + RT * kWaves - 1) / (RT * kWaves))), dim3(kThreads), st, Timing{}, a, columns, chunk);
}

template <bool BF16>
void launch(const MatvecArgs& args, hipStream_t st) {
    constexpr int PLANES = BF16 ? 1 : 3, kMost = BF16 ? 64 : 21;  // rows of x of which a line fits into LDS
    const int lines = (args.d + kLine - 1) / kLine;
    const int64_t tiles = (args.m + 15) / 16;
    // A wavefront of the wide kernel goes through whole rows, which takes its time however few
    // there are; the narrow one's wavefronts share a row, but not x.  us, narrow / wide, bf16,
    // 1 and 16 rows of x: m = 4096, d = 4096, 6.8 / 13.2 and 8.3 / 15.3; 8192, 10.3 / 13.5 and
    // 15.3 / 15.5; 12288, 13.5 / 13.7 and 21.1 / 15.9; 32768, 25.5 / 15.4 and 52.5 / 18.0; d =
    // 16384, m = 8192, 29.2 / 45.1 and 53.5 / 56.0; d = 2048, m = 8192, 6.4 / 8.3 and 8.2 / 9.1,
    // 10000, 7.8 / 8.3 and 10.8 / 9.1, 16384, 9.4 / 8.5 and 13.5 / 9.3; d = 4096, 64 rows, m =
    // 2048, 15.0 / 30.6, 8192, 54.9 / 33.5.
    if (tiles * ((args.rows + 15) / 16) < 640) {
        // as many wavefronts as have a line each, unless the tiles alone are many
        const int waves = (int)std::min<int64_t>(std::min(kNarrowWaves, lines), std::max<int64_t>(2, 8192 / tiles));
        launch_kernel(matvec_narrow_kernel<BF16>, dim3((unsigned)tiles, (args.rows + 15) / 16), dim3(64 * waves), st, Timing{}, args);
        return;
    }
    for (int t = 0; t < args.rows; t += kMost) {
        MatvecArgs a = args;
        a.rows = std::min(kMost, args.rows - t);
        a.row0 = t;
        // two tiles a wavefront where they leave two workgroups for each CU
        if (a.rows > 32)
            launch_wide<PLANES, 1, BF16 ? 4 : 2>(a, st);
        else if (a.rows > 16)
            launch_wide<PLANES, 1, 2>(a, st);
        else if (tiles >= 8192)
            launch_wide<PLANES, 2, 1>(a, st);
        else
            launch_wide<PLANES, 1, 1>(a, st);
    }
}

}  // namespace

hipError_t launch_matvec(const MatvecArgs& a, hipStream_t st) {
    if (a.bf16)
        launch<true>(a, st);
    else
        launch<false>(a, st);
    return hipGetLastError();
}

}  // namespace cmoe
