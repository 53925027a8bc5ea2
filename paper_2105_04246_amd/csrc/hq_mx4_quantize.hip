// Microscaled 4-bit quantization (hq_mx4_quantize, hq_mx4_quantize_sr) and its inverse (hq_mx4_dequantize).
//
//   block of 32 values x along an axis:  byte = max(exponent field of max |x| - 2 [+ 1 if its mantissa > 1.5: stochastic], 0)
//   t = |x| 2^(127 - byte), exact in fp32; code = t to nearest even on the grid 0 .. 6, or up with probability of t's share of its step
//
// Bound by HBM: 4 or 2 bytes read per value, 17/32 of a byte written per direction; stochastic rounding by the vector pipes (a draw's four integer
// multiplications at a quarter of the rate, one of them the term of the index's high word, made for every value; a rounding per direction).
// Each direction by workgroups of its own, in small pieces: along the rows 4 rows of 256 columns a wavefront, four columns a lane (a
// block lies in eight neighbouring lanes: three DPP steps find its maximum), along the columns 32 rows of 64 columns, a column a lane, whose block is
// the lane's own.  Eight wavefronts make the 256 rows of a chunk along the columns; its codes are put together in LDS, so that the container is
// written in whole 128-byte lines.  Large tensors, to nearest: both directions from one reading, 32 rows of 256 columns a wavefront
// whose values stay in registers (fp32: all 256 of a lane, and one is spilled).
// Measured, both directions (pieces / one reading, us): fp32 512 x 512 3.6 / 8.5, 2048 x 2048 5.0 / 9.3, 4096 x 2048 12.6 / 11.3, 16384 x 4096
// 88 / 75.5; bf16 4096 x 2048 7.9 / 10.1, 4096 x 4096 15.1 / 12.8, 16384 x 4096 52.7 / 49.2 (4.2 TB/s).  Stochastic: pieces throughout,
// fp32 512 x 512 5.8 / 26, 16384 x 4096 128 / 157.
// One direction alone, pieces (16384 x 4096, along the rows / along the columns, us; the input partly in the last-level cache from the call before):
// fp32 45 / 47.5, bf16 29 / 26.
#include "hq_internal.h"
#include "hq_mx4.h"

#include <algorithm>

namespace {

constexpr int MQ_WAVES = 8;
constexpr int MQ_PITCH = MX_CODES + 16;            // LDS row of a column's codes: 8 lanes' 16-byte stores fall into different banks

struct QuantizeArgs {
    const void *X;
    const int *offs;
    uint8_t *Q, *S, *Qt, *St;
    int rows, cols, segments;
    int kc;                                        // chunks along the columns' axis (of a row)
    int tiles_rows, tiles_cols;                    // row tiles of a matrix (without offs) of the workgroups along the rows, along the columns
    unsigned first_cols;                           // first workgroup along the columns, where they are others
    unsigned first;                                // the launch's first workgroup
    HqSr sr;
};

// A lane's values of one row, as loaded: four columns, or one.
template <int TYPE, int CPL> struct Loaded { typedef int T; };
template <> struct Loaded<HQ_FP32, 4> { typedef v4i T; };
template <> struct Loaded<HQ_BF16, 4> { typedef v2i T; };
template <> struct Loaded<HQ_FP16, 4> { typedef v2i T; };

template <int TYPE, int CPL> __device__ inline float loaded_value(const typename Loaded<TYPE, CPL>::T &v, int j)
{
    if constexpr (CPL == 1) return TYPE == HQ_FP32 ? __int_as_float(v) : HqReal<TYPE>::load((typename HqReal<TYPE>::T)v);
    else if constexpr (TYPE == HQ_FP32) return __int_as_float(v[j]);
    else return HqReal<TYPE>::load((unsigned short)((unsigned)v[j >> 1] >> (16 * (j & 1))));
}

typedef unsigned short v2us __attribute__((ext_vector_type(2)));
__device__ inline int pk_max_u16(int a, int b)
{
    return __builtin_bit_cast(int, __builtin_elementwise_max(__builtin_bit_cast(v2us, a), __builtin_bit_cast(v2us, b)));
}

// fp32 bits of a magnitude held as its type's own bits (they order like the magnitudes; infinities and NaN on top).
template <int TYPE> __device__ inline unsigned magnitude_bits(unsigned m)
{
    if constexpr (TYPE == HQ_FP32) return m;
    else return __float_as_uint(HqReal<TYPE>::load((unsigned short)m));
}

struct BlockScale {
    int byte;
    float unit;                                    // nearest: 2^(byte - 127); stochastic: 2^(127 - byte)
    int mask;                                      // 0 for a block that is not finite
};
template <bool SR> __device__ inline BlockScale block_scale(unsigned bits)
{
    const bool finite = bits < 0x7f800000u;
    int byte = (int)(bits >> 23) - 2;
    if (SR) byte += (bits & 0x7fffffu) > 0x400000u;
    byte = max(byte, 0);
    BlockScale s;
    s.byte = finite ? byte : 255;
    if (SR) s.unit = __int_as_float(finite ? (254 - byte) << 23 : 0);
    else    s.unit = __int_as_float(byte ? byte << 23 : 0x400000);      // (2^-127 is below the smallest normal number)
    s.mask = finite ? -1 : 0;
    return s;
}

// x to the grid value below or above it, in units of the block's scale; u: 24 random bits / 2^24.  (Infinities and NaN: masked by the caller.)
__device__ inline float stochastic_value(float x, float factor, float u)
{
    const float t = __fmul_rn(fabsf(x), factor);
    // steps are 0.5 below 2, 1 below 4, 2 from there on: half of the power of two below t, which counts from 1
    const int power = max(__float_as_int(t), 0x3f800000) & 0x7f800000;
    const float q = __fmul_rn(t, __int_as_float(0x7f800000 - power)), low = floorf(q);
    const float v = __fmul_rn(__fsub_rn(q, low) > u ? __fadd_rn(low, 1.0f) : low, __int_as_float(power - 0x800000));
    return copysignf(v, x);
}

// The workgroup's piece: WR rows a wavefront, CPL columns a lane.  `block`: its number among those of its kind.
template <int TYPE, bool ROWS, bool COLS, bool SR, int WR, int CPL>
__device__ inline void quantize_piece(const QuantizeArgs &a, unsigned block, uint8_t *lds)
{
    typedef typename HqReal<TYPE>::T T;
    typedef typename Loaded<TYPE, CPL>::T F;
    constexpr int NW = MQ_WAVES, TILE = WR * NW, WIDTH = 64 * CPL;
    static_assert(!COLS || TILE == MX_CHUNK, "a workgroup makes whole chunks along the columns");
    static_assert(!ROWS || WIDTH == MX_CHUNK, "a wavefront makes whole chunks along the rows");
    uint8_t *codes = lds, *col_scales = lds + (COLS ? WIDTH * MQ_PITCH : 0), *row_scales = col_scales + (COLS ? WIDTH * MX_SCALES : 0);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned across = ((unsigned)a.cols + WIDTH - 1) / WIDTH, y = block / across;
    const int c = (int)(block - y * across);

    int r0, valid;                                 // the workgroup's rows
    size_t matrix = 0;
    if (a.offs) {
        const HqSegment s = hq_segment_of<TILE>(a.offs, a.segments, a.rows, (int)y);
        if (s.e < 0) return;                       // (the same for all wavefronts)
        r0 = s.first + s.unit * TILE;
        valid = min(TILE, s.end - r0);
    } else {
        const unsigned tiles = (unsigned)(COLS ? a.tiles_cols : a.tiles_rows);
        matrix = y / tiles;
        r0 = (int)(y - (unsigned)matrix * tiles) * TILE;
        valid = min(TILE, a.rows - r0);
    }
    const int rw = r0 + WR * wave, vw = min(max(valid - WR * wave, 0), WR);
    const int c0 = c * WIDTH + CPL * lane, nc = min(max(a.cols - c0, 0), CPL);

    // ---- WR rows x CPL columns per lane
    F raw[WR];
    const size_t first = (matrix * (size_t)a.rows + (size_t)rw) * (size_t)a.cols + (size_t)c0;      // linear index of the lane's first value
    const T *row0 = static_cast<const T *>(a.X) + ((matrix * (size_t)a.rows + (size_t)rw) * (size_t)a.cols + (size_t)c * WIDTH);   // (uniform)
    const unsigned at = CPL * lane;
    if (vw > 0 && nc == CPL) {
#pragma unroll
        for (int r = 0; r < WR; r++) {
            const T *from = row0 + (size_t)min(r, vw - 1) * (size_t)a.cols + at;
            if constexpr (CPL == 1) raw[r] = TYPE == HQ_FP32 ? *reinterpret_cast<const int *>(from) : (int)*reinterpret_cast<const unsigned short *>(from);
            else __builtin_memcpy(&raw[r], __builtin_assume_aligned(from, sizeof(T)), sizeof(F));
        }
    } else {
#pragma unroll
        for (int r = 0; r < WR; r++) {
            if constexpr (CPL == 1) raw[r] = 0;
            else {
                T v[4] = {};
                if (r < vw)
                    for (int j = 0; j < nc; j++) v[j] = (row0 + (size_t)r * (size_t)a.cols)[at + j];
                __builtin_memcpy(&raw[r], v, sizeof(F));
            }
        }
    }
    if (vw < WR) {
#pragma unroll
        for (int r = 0; r < WR; r++) {
            if constexpr (CPL == 1) raw[r] = r < vw ? raw[r] : 0;
            else
#pragma unroll
                for (int k = 0; k < (int)(sizeof(F) / 4); k++) raw[r][k] = r < vw ? raw[r][k] : 0;
        }
    }

    // ---- scales along the columns: a block is a lane's own
    BlockScale cs[CPL];
    if (COLS) {
        unsigned m[CPL] = {};
        if constexpr (CPL == 1) {
#pragma unroll
            for (int r = 0; r < WR; r++) m[0] = max(m[0], (unsigned)raw[r] & (TYPE == HQ_FP32 ? 0x7fffffffu : 0x7fffu));
        } else if constexpr (TYPE == HQ_FP32) {
#pragma unroll
            for (int r = 0; r < WR; r++)
#pragma unroll
                for (int j = 0; j < 4; j++) m[j] = max(m[j], (unsigned)raw[r][j] & 0x7fffffffu);
        } else {
            int p[2] = {};
#pragma unroll
            for (int r = 0; r < WR; r++)
#pragma unroll
                for (int k = 0; k < 2; k++) p[k] = pk_max_u16(p[k], raw[r][k] & 0x7fff7fff);
#pragma unroll
            for (int j = 0; j < 4; j++) m[j] = ((unsigned)p[j >> 1] >> (16 * (j & 1))) & 0xffffu;
        }
#pragma unroll
        for (int j = 0; j < CPL; j++) {
            cs[j] = block_scale<SR>(magnitude_bits<TYPE>(m[j]));
            col_scales[(CPL * lane + j) * MX_SCALES + wave] = (uint8_t)cs[j].byte;
        }
    }

    // ---- codes, two rows at a time
    unsigned cc[CPL][4] = {};                      // codes along the columns: 32 rows of the lane's columns
    uint8_t *out = nullptr;
    if (ROWS) {
        // an even lane stores the codes of the even row for itself and its neighbour, an odd lane those of the odd row
        const size_t row = (matrix * (size_t)a.kc + (size_t)c) * (size_t)a.rows + (size_t)rw;
        out = a.Q + (row + (lane & 1)) * MX_CODES + (lane >> 1) * 4;
    }
    const unsigned pick = lane & 1 ? 0x03020706u : 0x05040100u;           // bytes of (neighbour's: 4 .. 7, own: 0 .. 3)
#pragma unroll
    for (int r = 0; r < WR; r += 2) {
        unsigned both = 0;
        float x[2][CPL], u[2][CPL];
#pragma unroll
        for (int i = 0; i < 2; i++) {
#pragma unroll
            for (int j = 0; j < CPL; j++) x[i][j] = loaded_value<TYPE, CPL>(raw[r + i], j);
            if (SR) {
                const size_t idx = first + (size_t)(r + i) * (size_t)a.cols;
#pragma unroll
                for (int j = 0; j < CPL; j++) {
                    const unsigned bits = hq_sr_bits((unsigned)(idx + j), (unsigned)((idx + j) >> 32) * 0x85ebca77u + a.sr.k1, a.sr.k0);
                    u[i][j] = __fmul_rn((float)(bits >> 8), 1.0f / 16777216.0f);
                }
            }
            if constexpr (ROWS) {
                unsigned m;
                if constexpr (TYPE == HQ_FP32) {
                    m = max(max((unsigned)raw[r + i][0] & 0x7fffffffu, (unsigned)raw[r + i][1] & 0x7fffffffu),
                            max((unsigned)raw[r + i][2] & 0x7fffffffu, (unsigned)raw[r + i][3] & 0x7fffffffu));
                } else {
                    const unsigned p = (unsigned)pk_max_u16(raw[r + i][0] & 0x7fff7fff, raw[r + i][1] & 0x7fff7fff);
                    m = max(p & 0xffffu, p >> 16);
                }
                m = (unsigned)hq_row_reduce<8>((int)m, HqMax());
                const BlockScale rs = block_scale<SR>(magnitude_bits<TYPE>(m));
                unsigned code = 0;
                if (SR) {
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) v[j] = stochastic_value(x[i][j], rs.unit, u[i][j]);
                    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], 1.0f, 0);
                    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], 1.0f, 1);
                } else {
                    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[i][0], x[i][1], rs.unit, 0);
                    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[i][2], x[i][3], rs.unit, 1);
                }
                both |= ((code & (unsigned)rs.mask) & 0xffffu) << (16 * i);
                if ((lane & 7) == 0) row_scales[(wave * WR + r + i) * MX_SCALES + (lane >> 3)] = (uint8_t)rs.byte;
            }
        }
        if (ROWS) {
            const unsigned other = (unsigned)hq_lane_partner<1>((int)both);
            const unsigned w = __builtin_amdgcn_perm(other, both, pick);
            if (r + (lane & 1) < vw) *reinterpret_cast<unsigned *>(out + r * MX_CODES) = w;
        }
        if (COLS) {
#pragma unroll
            for (int j = 0; j < CPL; j++) {
                const float v0 = SR ? stochastic_value(x[0][j], cs[j].unit, u[0][j]) : x[0][j];
                const float v1 = SR ? stochastic_value(x[1][j], cs[j].unit, u[1][j]) : x[1][j];
                const float unit = SR ? 1.0f : cs[j].unit;
                unsigned &d = cc[j][r / 8];
                switch (r % 8 / 2) {               // (the byte is part of the instruction)
                case 0: d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, v0, v1, unit, 0); break;
                case 1: d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, v0, v1, unit, 1); break;
                case 2: d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, v0, v1, unit, 2); break;
                default: d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, v0, v1, unit, 3); break;
                }
            }
        }
    }
    if (COLS) {
        // column CPL * lane + j is row j * 64 + lane of the LDS tile
#pragma unroll
        for (int j = 0; j < CPL; j++)
            *reinterpret_cast<v4i *>(codes + (j * 64 + lane) * MQ_PITCH + 16 * wave) =
                v4i{(int)cc[j][0] & cs[j].mask, (int)cc[j][1] & cs[j].mask, (int)cc[j][2] & cs[j].mask, (int)cc[j][3] & cs[j].mask};
    }
    __syncthreads();
    if (ROWS) {
        // WR rows x 8 bytes of a wavefront: one run
        const size_t row = (matrix * (size_t)a.kc + (size_t)c) * (size_t)a.rows + (size_t)rw;
        if ((lane >> 1) < vw)
            *reinterpret_cast<unsigned *>(a.S + row * MX_SCALES + 4 * lane) = *reinterpret_cast<const unsigned *>(row_scales + wave * WR * MX_SCALES + 4 * lane);
    }
    if (COLS) {
        const int ncols = min(a.cols - c * WIDTH, WIDTH);
        const size_t col = (size_t)y * (size_t)a.cols + (size_t)c * WIDTH;
        for (int k = threadIdx.x; k < ncols * (MX_CODES / 16); k += 64 * NW) {
            const int n = k >> 3, part = k & 7;
            *reinterpret_cast<v4i *>(a.Qt + (col + n) * MX_CODES + 16 * part) =
                *reinterpret_cast<const v4i *>(codes + (n % CPL * 64 + n / CPL) * MQ_PITCH + 16 * part);
        }
        for (int k = threadIdx.x; k < ncols * (MX_SCALES / 4); k += 64 * NW)
            *reinterpret_cast<unsigned *>(a.St + col * MX_SCALES + 4 * k) = *reinterpret_cast<const unsigned *>(col_scales + 4 * k);
    }
}

template <int CPL> constexpr int MQ_LDS_COLS = 64 * CPL * (MQ_PITCH + MX_SCALES);

// Both directions from one reading, to nearest.
template <int TYPE> __global__ __launch_bounds__(64 * MQ_WAVES) void mx4_quantize_kernel(const QuantizeArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[MQ_LDS_COLS<4> + MQ_WAVES * 32 * MX_SCALES];
    quantize_piece<TYPE, true, true, false, 32, 4>(a, a.first + blockIdx.x, lds);
}
// Each direction by workgroups of its own: along the rows up to a.first_cols, along the columns from there on.
template <int TYPE, bool SR> __global__ __launch_bounds__(64 * MQ_WAVES) void mx4_quantize_pieces_kernel(const QuantizeArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[MQ_LDS_COLS<1>];
    const unsigned block = a.first + blockIdx.x;
    if (block < a.first_cols) quantize_piece<TYPE, true, false, SR, 4, 4>(a, block, lds);
    else                      quantize_piece<TYPE, false, true, SR, 32, 1>(a, block - a.first_cols, lds);
}

// ---------------------------------------------------------------------------------------
struct DequantizeArgs {
    const uint8_t *Q, *S;
    const int *offs;
    void *X;
    int rows, n, segments;
    int chunks;                                    // of a matrix (without offs)
    int tiles;                                     // row tiles
    unsigned first;                                // the launch's first workgroup
};

template <int TYPE> constexpr int MD_ROWS = TYPE == HQ_FP32 ? 8 : 16;        // rows of a workgroup, in two turns; a lane writes 16 bytes of a row

template <int TYPE> __global__ __launch_bounds__(HQ_THREADS) void mx4_dequantize_kernel(const DequantizeArgs a)
{
    typedef typename HqReal<TYPE>::T T;
    const unsigned block = a.first + blockIdx.x, y = block / (unsigned)a.tiles;
    const int tile = (int)(block - y * (unsigned)a.tiles);
    int k0, valid;                                 // the chunk's place on the axis, its values
    size_t matrix = 0;
    if (a.offs) {
        const HqSegment s = hq_segment_of<MX_CHUNK>(a.offs, a.segments, a.n, (int)y);
        if (s.e < 0) return;
        k0 = s.first + s.unit * MX_CHUNK;
        valid = min(MX_CHUNK, s.end - k0);
    } else {
        matrix = y / (unsigned)a.chunks;
        k0 = (int)(y - (unsigned)matrix * (unsigned)a.chunks) * MX_CHUNK;
        valid = min(MX_CHUNK, a.n - k0);
    }
    constexpr int COUNT = 16 / sizeof(T), LANES = MX_CHUNK / COUNT;      // values of a lane, lanes of a row
    const int part = threadIdx.x % LANES, have = min(max(valid - COUNT * part, 0), COUNT);
    for (int r = tile * MD_ROWS<TYPE> + threadIdx.x / LANES; r < min(a.rows, (tile + 1) * MD_ROWS<TYPE>); r += HQ_THREADS / LANES) {
        const size_t row = (size_t)y * (size_t)a.rows + (size_t)r;
        unsigned code = 0;
        __builtin_memcpy(&code, __builtin_assume_aligned(a.Q + row * MX_CODES + COUNT / 2 * part, COUNT / 2), COUNT / 2);
        const unsigned byte = a.S[row * MX_SCALES + COUNT * part / HQ_MX4_BLOCK];
        const float scale = __uint_as_float(byte == 255 ? 0x7fc00000u : byte ? byte << 23 : 0x400000u);
        T v[COUNT];
        auto two = [&](v2f p, int k) __attribute__((always_inline)) {
            v[k] = HqReal<TYPE>::store(__fmul_rn(p[0], scale)); v[k + 1] = HqReal<TYPE>::store(__fmul_rn(p[1], scale));
        };
        two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 0), 0);
        two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 1), 2);
        if constexpr (COUNT == 8) {
            two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 2), 4);
            two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, 1.0f, 3), 6);
        }
        T *dst = static_cast<T *>(a.X) + (matrix * (size_t)a.rows + (size_t)r) * (size_t)a.n + (size_t)(k0 + COUNT * part);
        if (have == COUNT) {
            v4i x;
            __builtin_memcpy(&x, v, 16);
            __builtin_nontemporal_store((HqUnaligned16)x, reinterpret_cast<HqUnaligned16 *>(dst));
        } else
#pragma unroll
            for (int j = 0; j < COUNT; j++)
                if (j < have) dst[j] = v[j];
    }
}

inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

template <int TYPE> int launch_quantize(QuantizeArgs a, bool pieces, bool sr, unsigned blocks, hipStream_t s)
{
    constexpr unsigned threads = 64 * MQ_WAVES;
    return hq_mx4_launch(blocks, threads, [&](unsigned first, unsigned count) {
        a.first = first;
        if (!pieces) hipLaunchKernelGGL(mx4_quantize_kernel<TYPE>, dim3(count), dim3(threads), 0, s, a);
        else if (sr) hipLaunchKernelGGL((mx4_quantize_pieces_kernel<TYPE, true>), dim3(count), dim3(threads), 0, s, a);
        else         hipLaunchKernelGGL((mx4_quantize_pieces_kernel<TYPE, false>), dim3(count), dim3(threads), 0, s, a);
    });
}

int quantize(int32_t xtype, const void *X, int32_t rows, int32_t cols, int32_t batch, const int32_t *offs, const uint64_t *seed,
             uint8_t *Q, uint8_t *S, uint8_t *Qt, uint8_t *St, void *stream)
{
    if (!hq_mx4_type_ok(xtype) || (!Q != !S) || (!Qt != !St) || (!Q && !Qt)) return HQ_E_BADARG;
    if (rows < 0 || cols < 1 || batch < 1 || rows >= MX_MOST || cols >= MX_MOST || (offs && batch > HQ_MX4_MAX_SEGMENTS)) return HQ_E_BADSHAPE;
    if (misaligned(X, 16) || misaligned(Q, 16) || misaligned(S, 16) || misaligned(Qt, 16) || misaligned(St, 16) || misaligned(offs, 4)) return HQ_E_BADARG;
    QuantizeArgs a = {};
    a.X = X; a.offs = offs; a.Q = Q; a.S = S; a.Qt = Qt; a.St = St;
    a.rows = rows; a.cols = cols; a.segments = batch;
    a.kc = (int)hq_mx4_chunks(cols, 1);
    // row tiles of all matrices or segments (as hq_mx4_chunks: each may end with a part of one)
    auto row_tiles = [&](int tile) { return offs ? (long)((rows - std::min(batch, rows)) / tile + std::min(batch, rows)) : (long)((rows + tile - 1) / tile) * batch; };
    constexpr int PIECE_ROWS = 4 * MQ_WAVES;
    const long y = row_tiles(MX_CHUNK);
    a.tiles_cols = (rows + MX_CHUNK - 1) / MX_CHUNK;
    a.tiles_rows = (rows + PIECE_ROWS - 1) / PIECE_ROWS;
    if ((double)y * a.kc >= 2147483648.0) return HQ_E_BADSHAPE;
    const double along_rows = Q ? (double)row_tiles(PIECE_ROWS) * a.kc : 0, along_cols = Qt ? (double)y * ((cols + 63) / 64) : 0;
    // one reading: from 32 MB on (figures at the top)
    const bool pieces = !Q || !Qt || seed || (double)rows * cols * (offs ? 1 : batch) * hq_mx4_type_bytes(xtype) < 32 * 1048576.0;
    if (pieces && along_rows + along_cols >= 2147483648.0) return HQ_E_BADSHAPE;
    a.first_cols = (unsigned)along_rows;
    if (y == 0) return HQ_OK;
    if (!X) return HQ_E_BADARG;
    if (seed) a.sr = HqSr{(unsigned)*seed, (unsigned)(*seed >> 32)};
    const unsigned blocks = pieces ? (unsigned)(along_rows + along_cols) : (unsigned)(y * a.kc);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    switch (xtype) {
    case HQ_FP32: return launch_quantize<HQ_FP32>(a, pieces, seed, blocks, s);
    case HQ_BF16: return launch_quantize<HQ_BF16>(a, pieces, seed, blocks, s);
    default:      return launch_quantize<HQ_FP16>(a, pieces, seed, blocks, s);
    }
}

} // namespace

extern "C" {

int64_t hq_mx4_chunks(int64_t n, int32_t segments)
{
    if (n < 0 || n >= MX_MOST || segments < 1 || segments > HQ_MX4_MAX_SEGMENTS) return 0;
    // a first value opens a chunk for every segment that has one; of the rest, every 256 more open another
    const int64_t used = std::min<int64_t>(segments, n);
    return (n - used) / MX_CHUNK + used;
}

int hq_mx4_quantize(int32_t xtype, const void *X, int32_t rows, int32_t cols, int32_t batch, const int32_t *offs,
                    uint8_t *Q, uint8_t *S, uint8_t *Qt, uint8_t *St, void *stream)
{
    return quantize(xtype, X, rows, cols, batch, offs, nullptr, Q, S, Qt, St, stream);
}

int hq_mx4_quantize_sr(int32_t xtype, const void *X, int32_t rows, int32_t cols, int32_t batch, const int32_t *offs,
                       uint64_t seed, uint8_t *Q, uint8_t *S, uint8_t *Qt, uint8_t *St, void *stream)
{
    return quantize(xtype, X, rows, cols, batch, offs, &seed, Q, S, Qt, St, stream);
}

int hq_mx4_dequantize(const uint8_t *Q, const uint8_t *S, int32_t rows, int32_t n, int32_t batch, const int32_t *offs,
                      int32_t xtype, void *X, void *stream)
{
    if (!hq_mx4_type_ok(xtype)) return HQ_E_BADARG;
    if (rows < 0 || n < 0 || batch < 1 || rows >= MX_MOST || n >= MX_MOST || (offs && batch > HQ_MX4_MAX_SEGMENTS)) return HQ_E_BADSHAPE;
    if (misaligned(X, 16) || misaligned(Q, 16) || misaligned(S, 16) || misaligned(offs, 4)) return HQ_E_BADARG;
    DequantizeArgs a = {};
    a.Q = Q; a.S = S; a.offs = offs; a.X = X; a.rows = rows; a.n = n; a.segments = batch;
    a.chunks = (int)hq_mx4_chunks(n, 1);
    const int tile = xtype == HQ_FP32 ? MD_ROWS<HQ_FP32> : MD_ROWS<HQ_BF16>;
    a.tiles = (rows + tile - 1) / tile;
    const long y = offs ? (long)hq_mx4_chunks(n, batch) : (long)a.chunks * batch;
    if ((double)y * a.tiles >= 2147483648.0) return HQ_E_BADSHAPE;
    if (y == 0 || a.tiles == 0) return HQ_OK;
    if (!Q || !S || !X) return HQ_E_BADARG;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return hq_mx4_launch((unsigned)(y * a.tiles), HQ_THREADS, [&](unsigned first, unsigned count) {
        a.first = first;
        const dim3 grid(count), threads(HQ_THREADS);
        switch (xtype) {
        case HQ_FP32: hipLaunchKernelGGL(mx4_dequantize_kernel<HQ_FP32>, grid, threads, 0, s, a); break;
        case HQ_BF16: hipLaunchKernelGGL(mx4_dequantize_kernel<HQ_BF16>, grid, threads, 0, s, a); break;
        default:      hipLaunchKernelGGL(mx4_dequantize_kernel<HQ_FP16>, grid, threads, 0, s, a); break;
        }
    });
}

} // extern "C"
