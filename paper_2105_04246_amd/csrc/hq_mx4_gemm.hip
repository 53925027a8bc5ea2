// Products of microscaled 4-bit matrices: hq_mx4_gemm, hq_mx4_gemm_grouped (ragged rows by expert), hq_mx4_wgrad_grouped
// (ragged segments of the contraction).
//
//   out[m][n] = sum_blocks 2^(sa[m][b] + sb[n][b] - 254) sum_{k in b} a[m][k] b[n][k]
//
// on the scaled MFMA (16 x 16 x 128, fp4 x fp4): a lane holds one block of a row, 16 bytes, and its scale byte; the products are summed
// in fp32 by the matrix pipe.  (32 x 32 x 64 does the same work at more power: register-only loops on random codes sustain 6.2 PFLOP/s with it
// and 6.7 with this one; on codes of 0 9.7 and 9.4.)  Containers are cut along the contraction into chunks of 256 values, 128 bytes a row; the
// rows of a chunk follow each other, so a tile's operands of one chunk are one run of memory, at any row offset, and there is no tail along the
// contraction (behind its end the codes are 0).
#include "hq_internal.h"
#include "hq_mx4.h"

#include <algorithm>
#include <type_traits>

namespace {

enum { DENSE = 0, BY_ROWS = 1, BY_CHUNKS = 2 };   // one product; rows of A by expert; chunks of both by expert

struct ProductArgs {
    const uint8_t *A, *As, *B, *Bs;
    const int *offs;
    void *out;                     // split contractions: their partial sums [splits][outputs], fp32
    size_t outputs;
    int M, N;                      // rows of A and of out (BY_ROWS: of all experts together), rows of B
    int chunks;                    // of the contraction (BY_CHUNKS: the most that the segments can have)
    int rows;                      // BY_CHUNKS: values along the contraction in all segments
    int experts, splits;
    int m_tiles, n_tiles;
    int out_type;
    unsigned first;                // the launch's first workgroup
};

template <int SCALE_BYTE> __device__ inline v4f mfma16(v4i a, v4i b, v4f c, int sa, int sb)
{
    const v8i a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1), b8 = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, SCALE_BYTE, sa, SCALE_BYTE, sb);
}

// Before results of mfma16 go to LDS: the compiler (clang of ROCm 7.2) stored the first ones right behind the loop that makes them, without the
// wait states that the matrix pipe needs before its registers are read (it puts them before the second store).
__device__ inline void mfma16_done(v4f &c) { asm volatile("s_nop 15" : "+v"(c)); }

// COUNT consecutive outputs from column n on, of N, to `dst` (the address of column n); rounded once.
template <int TYPE, int COUNT> __device__ inline void store_run(void *dst, const float *v, int n, int N)
{
    typedef typename HqReal<TYPE>::T T;
    T *d = static_cast<T *>(dst);
    if (n + COUNT <= N) {
        T t[COUNT];
#pragma unroll
        for (int e = 0; e < COUNT; e++) t[e] = HqReal<TYPE>::store(v[e]);
        if constexpr (sizeof(t) == 16) {
            // (past L2, which the operands of the tiles to come are to stay in: weight gradients of 16 experts, 4096 x 1024 fp32 over 16384 rows,
            // 104 -> 81 us; forward pass of 8 experts, 8192 x 4096 bf16, 42 -> 39)
            v4i x;
            __builtin_memcpy(&x, t, 16);
            __builtin_nontemporal_store((HqUnaligned16)x, reinterpret_cast<HqUnaligned16 *>(d));
        } else __builtin_memcpy(__builtin_assume_aligned(d, sizeof(T)), t, sizeof(t));
    } else {
#pragma unroll
        for (int e = 0; e < COUNT; e++)
            if (n + e < N) d[e] = HqReal<TYPE>::store(v[e]);
    }
}

// ---------------------------------------------------------------------------------------
// Tiles of BM x BN outputs, WM x WN wavefronts of (BM / WM) x (BN / WN) each.  A stage is one chunk of the tile's rows of A and B, straight
// from memory into one of two LDS buffers.  A step is half a chunk: one of a lane's two blocks of a row.  Tiles of 256 have 8 wavefronts of 64 x 128
// (128 accumulator registers a lane, one workgroup to a compute unit), which read 192 KB of fragments a stage from LDS; tiles of 128 (4 wavefronts,
// two workgroups) and of 64 (2 wavefronts, four) fill the card where there are few.
// Measured: 8192 x 4096 x 4096 to bf16 64 us, 4.3 PFLOP/s (tiles of 128 86, of 64 121); the matrix pipes are busy for 46 % of the cycles at 2.07
// GHz, and for 21 % of them a compute unit has no wavefront.  Beside 66.5 us of the same run: without stores 60, without loads 59, without both 49;
// loads alone 38 (570 MB through L2), stores alone 14, none of the three 4.  (Codes of 0, which leave the clock higher: 54 us for 63.)  What holds it
// up is that the three overlap in part only: a compute unit has one workgroup, and two tiles, one after the other.  Slower (against 66 to 74 of the same day):
// stages of half a chunk in a ring of four 87 us, one buffer and four workgroups of 128 x 128 102, workgroups that keep their place and request the
// next tile's stages before they store 77 (with spilled registers), lines touched ahead of their loads 73.
// Weight gradients of 16 experts, 4096 x 1024 fp32 over 16384 rows: 63 to 65 us, 268 MB written and 60 MB read from memory (5.2 TB/s, a copy's rate).
// ---------------------------------------------------------------------------------------

// What the 16-byte blocks of an LDS row are XORed with.  Rows 2 k and 2 k + 1 take the two halves of the banks, the eight values of k all eight places of a
// half.  The pipe serves a 16-byte read in four turns of 16 lanes, rows 0 .. 3 and 12 .. 15 of one group of lanes with rows 4 .. 11 of the next one,
// whose blocks are 2 further on: the four places of k = 0, 1, 6, 7 are a set that XOR 2 maps onto itself, and so are the others.  (With k
// itself, 44 % of the LDS cycles were conflicts.)
__device__ inline int swizzle(int row)
{
    const int k = (row >> 1) & 7;
    return (k & 3) | (((k ^ (k >> 1)) & 2) << 1);
}

template <int BM, int BN, int WM, int WN, int GROUP>
__global__ __launch_bounds__(64 * WM * WN) void mx4_tile_kernel(const ProductArgs a)
{
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int CODE_LOADS = (BM + BN) / 8 / NW, SCALE_LOADS = (BM + BN) / 32 / NW;
    static_assert(BM % (32 * NW) == 0 && BN % (32 * NW) == 0, "a load of all wavefronts belongs to one operand");
    constexpr int STAGE = (BM + BN) * (MX_CODES + MX_SCALES);
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = lane >> 4, r16 = lane & 15, wm = wave / WN, wn = wave % WN;

    // ---- which tile: each XCD takes a run of them, in bands of row tiles
    const int per_split = a.m_tiles * a.n_tiles * (GROUP == BY_CHUNKS ? a.experts : 1);
    const unsigned block = a.first + blockIdx.x;
    const int split = block / per_split;
    int tile = block - split * per_split;
    const int per = per_split / 8;
    if (tile < per * 8) tile = (tile & 7) * per + (tile >> 3);
    int e = 0;
    if (GROUP == BY_CHUNKS) {
        // (every expert's tiles over all XCDs: their contractions differ in length)
        const int mn = a.m_tiles * a.n_tiles, share = mn / 8, b = block - split * per_split;
        if (share) {
            if (b < share * 8 * a.experts) {
                const int x = b & 7, t = b >> 3;
                e = t / share;
                tile = x * share + t - e * share;
            } else {
                const int t = b - share * 8 * a.experts, left = mn - 8 * share;
                e = t / left;
                tile = 8 * share + t - e * left;
            }
        } else { e = b / mn; tile = b - e * mn; }
    }
    // (tiles that run on an XCD together share operand panels: 4 x 8 of the largest.  8192 x 4096 x 4096 in bands of 8: 72 us, of 4: 68)
    constexpr int BAND = BM == 256 ? 4 : 8;
    const int band = tile / (BAND * a.n_tiles), in_band = min(BAND, a.m_tiles - BAND * band), rest = tile - band * BAND * a.n_tiles;
    const int tile_n = rest / in_band, tile_m = BAND * band + rest - tile_n * in_band;

    int m0 = tile_m * BM, m_end = a.M, chunk0 = 0, nst = a.chunks;
    const int n0 = tile_n * BN;
    size_t b_chunk0 = 0;
    if (GROUP == BY_ROWS) {
        const HqSegment s = hq_segment_of<BM>(a.offs, a.experts, a.M, tile_m);
        if (s.e < 0) return;
        m0 = s.first + s.unit * BM;
        m_end = s.end;
        b_chunk0 = (size_t)s.e * (size_t)a.chunks;
    } else if (GROUP == BY_CHUNKS) {
        const HqSegment s = hq_segment_start<MX_CHUNK>(a.offs, a.rows, e);
        chunk0 = min(max(s.unit, 0), a.chunks);
        nst = min((s.end - s.first + MX_CHUNK - 1) / MX_CHUNK, a.chunks - chunk0);
    }
    if (a.splits > 1) {
        const int from = (int)((long)nst * split / a.splits), to = (int)((long)nst * (split + 1) / a.splits);
        chunk0 += from;
        nst = to - from;
    }
    if (GROUP != BY_ROWS) b_chunk0 = (size_t)chunk0;

    // ---- loads: 8 rows of codes or 32 rows of scales each; rows past the end repeat the last (never stored)
    const uint8_t *code_a = a.A + ((size_t)chunk0 * (size_t)a.M + (size_t)m0) * MX_CODES, *scale_a = a.As + ((size_t)chunk0 * (size_t)a.M + (size_t)m0) * MX_SCALES;
    const uint8_t *code_b = a.B + (b_chunk0 * (size_t)a.N + (size_t)n0) * MX_CODES, *scale_b = a.Bs + (b_chunk0 * (size_t)a.N + (size_t)n0) * MX_SCALES;
    unsigned code_off[CODE_LOADS], scale_off[SCALE_LOADS];
    // Of a wavefront's columns, LDS row 16 * j + r holds this one, so that a lane has neighbours of 16 bytes and 16 lanes a run of 256.
    const bool wide = TN == 8 && a.out_type != HQ_FP32;
    auto column_of = [&](int j, int r) __attribute__((always_inline)) { return wide ? 8 * r + j : (j & ~3) * 16 + 4 * r + (j & 3); };
    auto row_of = [&](int row) __attribute__((always_inline)) {          // LDS row -> row of its operand, from the tile's first
        if (row < BM) return min(row, m_end - 1 - m0);
        const int c = row - BM, in = c % (16 * TN);
        return min(c - in + column_of(in >> 4, in & 15), a.N - 1 - n0);
    };
#pragma unroll
    for (int k = 0; k < CODE_LOADS; k++) {
        const int row = 8 * (NW * k + wave) + (lane >> 3);
        code_off[k] = (unsigned)row_of(row) * MX_CODES + 16u * (unsigned)((lane & 7) ^ swizzle(row));
    }
#pragma unroll
    for (int k = 0; k < SCALE_LOADS; k++) scale_off[k] = (unsigned)row_of(32 * (NW * k + wave) + (lane >> 1)) * MX_SCALES + 4u * (unsigned)(lane & 1);
    const unsigned lds0 = hq_lds_address(smem) + 1024 * wave, lds1 = hq_lds_address(smem) + (BM + BN) * MX_CODES + 256 * wave;
    auto request = [&](int buf, int k) __attribute__((always_inline)) {  // load k of the next stage
        if (k < CODE_LOADS)
            hq_lds_load16(reinterpret_cast<const int8_t *>(8 * NW * k < BM ? code_a : code_b), code_off[k], lds0 + buf * STAGE + 1024 * NW * k);
        else {
            const int q = k - CODE_LOADS;
            hq_lds_load4(32 * NW * q < BM ? scale_a : scale_b, scale_off[q], lds1 + buf * STAGE + 256 * NW * q);
        }
    };
    constexpr int LOADS = CODE_LOADS + SCALE_LOADS;
    auto requested = [&]() __attribute__((always_inline)) {
        code_a += (size_t)a.M * MX_CODES; scale_a += (size_t)a.M * MX_SCALES;
        code_b += (size_t)a.N * MX_CODES; scale_b += (size_t)a.N * MX_SCALES;
    };

    v4f acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    // Fragments of A are kept twice, those of B once: a step goes through them in turn and each is loaded for the next step when it has been used.
    v4i fa[2][TM], fb[TN];
    int sa[TM], sa_next[TM], sb[TN];
    const int row_a = wm * (BM / WM) + r16, row_b = BM + wn * (BN / WN) + r16;
    int cur = 0;
    auto codes_at = [&](int row, int step) __attribute__((always_inline)) {
        return *reinterpret_cast<const v4i *>(smem + cur * STAGE + 16 * ((2 * group + step) ^ swizzle(r16)) + row * MX_CODES);
    };
    auto scale_at = [&](int row) __attribute__((always_inline)) {
        return (int)*reinterpret_cast<const unsigned short *>(smem + cur * STAGE + (BM + BN) * MX_CODES + 2 * group + row * MX_SCALES);
    };
    if (nst > 0) {
#pragma unroll
        for (int k = 0; k < LOADS; k++) request(0, k);
        requested();
        if (nst > 1) {
#pragma unroll
            for (int k = 0; k < LOADS; k++) request(1, k);
            requested();
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
        } else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TM; i++) { fa[0][i] = codes_at(row_a + 16 * i, 0); sa[i] = scale_at(row_a + 16 * i); }
#pragma unroll
        for (int j = 0; j < TN; j++) { fb[j] = codes_at(row_b + 16 * j, 0); sb[j] = scale_at(row_b + 16 * j); }
    }
    // `next`: there is a stage after this one; `more`: and another one.  (Nothing moves across the lines; no branches, which the compiler would
    // let products sink below.)
    auto stage = [&](auto more, auto next) __attribute__((always_inline)) {
        constexpr bool MORE = decltype(more)::value, NEXT = decltype(next)::value;
#pragma unroll
        for (int j = 0; j < TN; j++) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < TM; i++) acc[i][j] = mfma16<0>(fa[0][i], fb[j], acc[i][j], sa[i], sb[j]);
            __builtin_amdgcn_sched_barrier(0);
            if (j < TM) fa[1][j] = codes_at(row_a + 16 * j, 1);
            fb[j] = codes_at(row_b + 16 * j, 1);
        }
        const int freed = cur;
        if (NEXT) {
            // all fragments of this stage are in registers at the barrier: its buffer takes the stage after next
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            cur ^= 1;
        }
#pragma unroll
        for (int j = 0; j < TN; j++) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < TM; i++) acc[i][j] = mfma16<1>(fa[1][i], fb[j], acc[i][j], sa[i], sb[j]);
            __builtin_amdgcn_sched_barrier(0);
            if (MORE) {
#pragma unroll
                for (int k = j * LOADS / TN; k < (j + 1) * LOADS / TN; k++) request(freed, k);
            }
            if (NEXT) {
                if (j < TM) { fa[0][j] = codes_at(row_a + 16 * j, 0); sa_next[j] = scale_at(row_a + 16 * j); }
                fb[j] = codes_at(row_b + 16 * j, 0);
                sb[j] = scale_at(row_b + 16 * j);
            }
        }
        if (MORE) requested();
        if (NEXT) {
#pragma unroll
            for (int i = 0; i < TM; i++) sa[i] = sa_next[i];
        }
    };
    int s = 0;
    for (; s + 2 < nst; s++) stage(std::true_type(), std::true_type());
    if (s + 1 < nst) { stage(std::false_type(), std::true_type()); s++; }
    if (s < nst) stage(std::false_type(), std::false_type());
    // (all loads have been waited for: no wavefront ends with one into LDS under way.  The wait states are those of mfma16_done.)
    asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15" ::: "memory");

    // ---- a lane's columns of a row, 16 bytes at a time
    auto finish = [&](auto type, void *out) __attribute__((always_inline)) {
        constexpr int TYPE = decltype(type)::value, RUN = TYPE == HQ_FP32 ? 4 : TN;
        typedef typename HqReal<TYPE>::T T;
        const int m = m0 + wm * (BM / WM) + 4 * group, n = n0 + wn * (BN / WN) + RUN * r16;
        T *dst = static_cast<T *>(out) + ((size_t)m * (size_t)a.N + (size_t)n);
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int k = 0; k < 4; k++)
#pragma unroll
                for (int j = 0; j < TN; j += RUN) {
                    float v[RUN];
#pragma unroll
                    for (int c = 0; c < RUN; c++) v[c] = acc[i][j + c][k];
                    if (m + 16 * i + k < m_end) store_run<TYPE, RUN>(dst + (size_t)(16 * i + k) * (size_t)a.N + 16 * j, v, n + 16 * j, a.N);
                }
    };
    const size_t first = (GROUP == BY_CHUNKS ? (size_t)e * (size_t)a.M * (size_t)a.N : 0) + (size_t)split * a.outputs;
    if (a.out_type == HQ_FP32) finish(std::integral_constant<int, HQ_FP32>(), static_cast<float *>(a.out) + first);
    else if (a.out_type == HQ_BF16) finish(std::integral_constant<int, HQ_BF16>(), static_cast<unsigned short *>(a.out) + first);
    else finish(std::integral_constant<int, HQ_FP16>(), static_cast<unsigned short *>(a.out) + first);
}

// ---------------------------------------------------------------------------------------
// Few rows: the bytes of B and latency count.  A workgroup takes 16 rows of B (of one expert) and all rows of A that meet them, 16 * MT at a time;
// its wavefronts share the chunks between them and are added in LDS, in order.  Fragments come straight from memory, a lane 32 bytes of a row: the
// rows of a chunk follow each other, so a wavefront reads runs of 2 KB.
// Measured: 1 row, 4096 x 4096 3.7 to 4.0 us (8.9 MB of B: 2.2 TB/s and more, of which 2 us are an empty launch's); 16 rows, 32 experts of 2048 x 1024
// 5.0 us (3.5 TB/s).
// ---------------------------------------------------------------------------------------
template <int MT, int GROUP> __global__ __launch_bounds__(512) void mx4_row_kernel(const ProductArgs a)
{
    __shared__ float sums[8][MT][16][17];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int r16 = lane & 15, group = lane >> 4;
    const unsigned block = a.first + blockIdx.x;
    const int e = GROUP == BY_ROWS ? block / a.n_tiles : 0;
    const int n0 = (int)(block - (unsigned)e * (unsigned)a.n_tiles) * 16;
    int m_first = 0, m_end = a.M;
    if (GROUP == BY_ROWS) {
        m_first = hq_segment_bound(a.offs, e, a.M);
        m_end = hq_segment_bound(a.offs, e + 1, a.M);
    }
    const size_t n = (size_t)min(n0 + r16, a.N - 1);
    const uint8_t *b = a.B + ((size_t)e * (size_t)a.chunks * (size_t)a.N + n) * MX_CODES + 32 * group;
    const uint8_t *bs = a.Bs + ((size_t)e * (size_t)a.chunks * (size_t)a.N + n) * MX_SCALES + 2 * group;
    for (int m0 = m_first; m0 < m_end; m0 += 16 * MT) {
        v4f acc[MT];
        size_t m[MT];
#pragma unroll
        for (int t = 0; t < MT; t++) {
            acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            m[t] = (size_t)min(m0 + 16 * t + r16, m_end - 1);
        }
        for (int c = wave; c < a.chunks; c += waves) {
            const uint8_t *bp = b + (size_t)c * (size_t)a.N * MX_CODES;
            const v4i b0 = *reinterpret_cast<const v4i *>(bp), b1 = *reinterpret_cast<const v4i *>(bp + 16);
            const int sb = *reinterpret_cast<const unsigned short *>(bs + (size_t)c * (size_t)a.N * MX_SCALES);
#pragma unroll
            for (int t = 0; t < MT; t++) {
                const size_t row = (size_t)c * (size_t)a.M + m[t];
                const uint8_t *ap = a.A + row * MX_CODES + 32 * group;
                const v4i a0 = *reinterpret_cast<const v4i *>(ap), a1 = *reinterpret_cast<const v4i *>(ap + 16);
                const int sa = *reinterpret_cast<const unsigned short *>(a.As + row * MX_SCALES + 2 * group);
                acc[t] = mfma16<0>(b0, a0, acc[t], sb, sa);
                acc[t] = mfma16<1>(b1, a1, acc[t], sb, sa);
            }
        }
        // (lane: row r16 of A, rows 4 * group .. + 3 of B)
#pragma unroll
        for (int t = 0; t < MT; t++) mfma16_done(acc[t]);
#pragma unroll
        for (int t = 0; t < MT; t++)
#pragma unroll
            for (int k = 0; k < 4; k++) sums[wave][t][r16][4 * group + k] = acc[t][k];
        __syncthreads();
        for (int k = threadIdx.x; k < MT * 256; k += blockDim.x) {
            const int row = m0 + (k >> 4), col = n0 + (k & 15);
            float v = 0.0f;
            for (int w = 0; w < waves; w++) v = __fadd_rn(v, sums[w][k >> 8][(k >> 4) & 15][k & 15]);
            if (row < m_end && col < a.N) {
                const size_t o = (size_t)row * (size_t)a.N + (size_t)col;
                if (a.out_type == HQ_FP32) static_cast<float *>(a.out)[o] = v;
                else if (a.out_type == HQ_BF16) static_cast<unsigned short *>(a.out)[o] = HqReal<HQ_BF16>::store(v);
                else static_cast<unsigned short *>(a.out)[o] = HqReal<HQ_FP16>::store(v);
            }
        }
        __syncthreads();
    }
}

// ---- partial sums of split contractions, added in order: WIDTH outputs a lane -------------
template <int TYPE, int WIDTH> __global__ __launch_bounds__(HQ_THREADS) void mx4_join_kernel(const float *part, size_t outputs, int splits, void *out)
{
    typedef typename HqReal<TYPE>::T T;
    typedef float V __attribute__((ext_vector_type(WIDTH)));
    for (size_t g = ((size_t)blockIdx.x * HQ_THREADS + threadIdx.x) * WIDTH; g < outputs; g += (size_t)gridDim.x * HQ_THREADS * WIDTH) {
        V v = *reinterpret_cast<const V *>(part + g);
#pragma unroll 4
        for (int s = 1; s < splits; s++) {
            const V x = *reinterpret_cast<const V *>(part + (size_t)s * outputs + g);
#pragma unroll
            for (int j = 0; j < WIDTH; j++) v[j] = __fadd_rn(v[j], x[j]);
        }
        T t[WIDTH];
#pragma unroll
        for (int j = 0; j < WIDTH; j++) t[j] = HqReal<TYPE>::store(v[j]);
        __builtin_memcpy(static_cast<T *>(out) + g, t, sizeof(t));
    }
}
template <int TYPE> void launch_join(const float *part, size_t outputs, int splits, void *out, hipStream_t s)
{
    const int width = outputs % 4 == 0 ? 4 : 1;                          // (16-byte loads of every partial sum)
    const unsigned blocks = (unsigned)std::min<size_t>((outputs / width + HQ_THREADS - 1) / HQ_THREADS, 8192);
    if (width == 4) hipLaunchKernelGGL((mx4_join_kernel<TYPE, 4>), dim3(blocks), dim3(HQ_THREADS), 0, s, part, outputs, splits, out);
    else            hipLaunchKernelGGL((mx4_join_kernel<TYPE, 1>), dim3(blocks), dim3(HQ_THREADS), 0, s, part, outputs, splits, out);
}

// ---------------------------------------------------------------------------------------
inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
inline int launch_status() { return hipGetLastError() == hipSuccess ? HQ_OK : HQ_E_HIP; }

int check_product(const hq_mx4_problem *p, bool grouped)
{
    if (!p) return HQ_E_BADARG;
    if (!hq_mx4_type_ok(p->out_type)) return HQ_E_BADARG;
    if (p->M < 0 || p->N < 0 || p->K < 0 || p->M >= MX_MOST || p->N >= MX_MOST || p->K >= MX_MOST) return HQ_E_BADSHAPE;
    if (p->experts < 1 || p->experts > (grouped ? HQ_MX4_MAX_SEGMENTS : 1)) return HQ_E_BADSHAPE;
    return HQ_OK;
}

struct Plan { int side, splits; };                 // side: 1, 2: few rows, 16 of them at a time or 32; otherwise the tile's side

int tiles_of(long n, int side) { return (int)((n + side - 1) / side); }

// Microseconds that a launch takes, so that tile and split can be chosen: a start, the stages of a workgroup, and the bytes of the outputs.  A
// stage takes its latency while the compute units hold all workgroups at once, from there on their share of the card.  Fitted to (this / measured, us)
// products to bf16 in tiles of 64, 128, 256: 256 x 4096 x 4096 11.3 / 10.5, 15.6 / 15.3, 20 / 22; 1024 x 4096 x 4096 18.3 / 16.7, 16.9 / 17.0,
// 24.3 / 23.2; 2048 x 4096 x 4096 34 / 33, 27.9 / 24.7, 30.0 / 25.7; 4096 x 4096 x 4096 65 / 62, 53 / 48, 43 / 36; 1024 x 1024 x 16384 four ways
// 25.4 / 23.3, 23.9 / 24.1, 31.3 / 30.3, one way 37 / 43, 54 / 60, 72 / 85.
// It adds the outputs' time to that of stages which run beside them, so it says too much where outputs are many (8192 x 4096 x 4096 83 / 64; weight gradients
// of 16 experts, 4096 x 1024 over 16384 rows, 92 / 63) and leans to smaller tiles there.  By expert, tiles of 64, 128, 256, us (*: what it takes;
// products: rows x outputs of a row x contraction):
//   products, 8 experts:  512 x 4096 x 1024    9.4*  9.9  10.7      products, 8 experts:   1024 x 1024 x 1024   6.1*  6.9   9.5
//                        1024                 13.3  11.6* 11.0                             4096                10.7   9.7* 10.2
//                        2048                 17.6  15.0* 13.8                             8192                15.7  15.0* 11.2
//                        4096                 28.0  22.2  22.3*                            8192 x 1024 x 4096  36.9  35.5* 24.7
//                        8192                 45.9  35.6  33.8*     products, 32 experts:  4096 x 1024 x 4096  30.7  27.4* 26.5
//                       16384                 84.3  62.9  56.7*                           16384 x 1024 x 1024  27.2  22.4  22.8*
//   weight gradients:  4096 x 1024, 16384 rows, 16 experts  96.9  76.2  71.1*      1024 x 1024, 8192 rows, 4 experts  10.7  12.4* 15.8
//                      4096 x 1024,  8192 rows, 16 experts  67.4  56.9  58.5*       512 x 512, 16384 rows, 8 experts  10.5* 10.2  14.9
//                      2048 x 1024, 16384 rows,  4 experts  34.6  25.6* 28.8        512 x 512,  4096 rows, 8 experts   5.5*  5.8   8.5
//                      1024 x 1024, 16384 rows,  8 experts  22.1  19.3* 19.4        256 x 512,  4096 rows, 4 experts   5.6*  7.1  10.5
//   split 1, 2, 4, 8 ways:  512 x 1024, 16384 rows, 2 experts  tiles of 64 19.8 17.9 17.5 24.8, of 128 28.0 20.8 18.2* 22.6
//                           256 x 512,  16384 rows, 2 experts  tiles of 64 18.2 13.9 12.0 12.9*, of 128 27.4 18.9 14.6 13.7
double estimate(int side, int splits, double tiles, double stages, double outputs, double bytes)
{
    const double n = tiles * splits;
    const double stage = side == 64 ? std::max(0.40 + 0.00047 * n, 0.00086 * n) : side == 128 ? std::max(0.79, 0.0027 * n) : std::max(1.0 + 0.0040 * n, 0.0082 * n);
    return 2.6 + stage * (stages / splits) + (splits > 1 ? 2.2 + splits * outputs * 8 / 5.2e6 : outputs * bytes / 5.2e6);
}

Plan plan_of(const hq_mx4_problem *p, int group)
{
    // Few rows: B is read once and the rows of A beside it, without LDS.  (Rows / tiles of 64, us: one product of K = 4096, N = 4096 16 rows
    // 4.3 / 9, 32 rows 5.3 / 8.5, 64 rows 9.2 / 9.1.  By expert the count is known on the device only, its mean here: 64 experts of 4096 x 1024
    // 128 rows 21.1 / 26.3, 512 rows 32.5 / 29.9; 8 experts of 1024 x 4096 32 rows 5.9 / 10.3, 128 rows 12.5 / 10.5; 2 experts 32 rows 5.1 / 10.4.)
    // A mean says nothing of the routing.  Just below and at the line, all rows with one expert (evenly): 64 experts of 4096 x 1024 39 / 25 (32 / 30);
    // 8 of 1024 x 4096 12.1 / 10.6 (5.7 / 10.5); 256 of 2048 x 1024 155 / 55 (66 / 75); 4096 of 256 x 512 2100 / 514 (69 / 493), its rows 16 at a time.
    const long experts = p->experts;
    if (group == BY_ROWS && p->M < 8 * experts) return Plan{1, 1};
    if (group != BY_CHUNKS && p->M <= 32) return Plan{p->M <= 16 ? 1 : 2, 1};
    const double outputs = (double)p->M * p->N * (group == BY_CHUNKS ? experts : 1), bytes = (double)hq_mx4_type_bytes(p->out_type);
    // (segments: half a unit more than their rows fill)
    const double stages = group == BY_CHUNKS ? (double)p->K / (256.0 * experts) + 0.5 : (double)hq_mx4_chunks(p->K, 1);
    Plan best = {64, 1};
    double least = 1e30;
    for (int side = 64; side <= 256; side *= 2) {
        const double m = group == BY_ROWS ? (double)p->M / side + 0.5 * std::min<long>(experts, p->M) : (double)tiles_of(p->M, side);
        const double tiles = m * tiles_of(p->N, side) * (group == BY_CHUNKS ? experts : 1);
        for (int splits = 1; splits == 1 || (group != BY_ROWS && splits <= 16 && stages / splits >= 2); splits *= 2) {
            const double us = estimate(side, splits, tiles, stages, outputs, bytes);
            if (us < least) { least = us; best = Plan{side, splits}; }
        }
    }
    return best;
}

size_t outputs_of(const hq_mx4_problem *p, int group)
{
    return (size_t)p->M * (size_t)p->N * (group == BY_CHUNKS ? (size_t)p->experts : 1);
}

template <int BM, int BN, int WM, int WN, int GROUP> int launch_tile(ProductArgs a, unsigned blocks, hipStream_t s)
{
    const size_t lds = 2 * (BM + BN) * (MX_CODES + MX_SCALES);
    static std::atomic<unsigned long long> allowed{0};
    if (!hq_allow_lds(mx4_tile_kernel<BM, BN, WM, WN, GROUP>, lds, allowed)) return HQ_E_HIP;
    return hq_mx4_launch(blocks, 64 * WM * WN, [&](unsigned first, unsigned count) {
        a.first = first;
        hipLaunchKernelGGL((mx4_tile_kernel<BM, BN, WM, WN, GROUP>), dim3(count), dim3(64 * WM * WN), lds, s, a);
    });
}

template <int GROUP> int product(const hq_mx4_problem *p, const uint8_t *A, const uint8_t *As, const uint8_t *B, const uint8_t *Bs,
                                 const int32_t *offs, void *out, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_product(p, GROUP != DENSE);
    if (rc != HQ_OK) return rc;
    if (misaligned(A, 16) || misaligned(As, 16) || misaligned(B, 16) || misaligned(Bs, 16) || misaligned(out, 16) || misaligned(offs, 4)) return HQ_E_BADARG;
    if (p->M == 0 || p->N == 0) return HQ_OK;
    if (!out || (GROUP != DENSE && !offs) || (p->K > 0 && (!A || !As || !B || !Bs))) return HQ_E_BADARG;
    const Plan plan = plan_of(p, GROUP);
    ProductArgs a = {};
    a.A = A; a.As = As; a.B = B; a.Bs = Bs; a.offs = offs; a.out = out;
    a.M = p->M; a.N = p->N; a.experts = p->experts; a.out_type = p->out_type;
    a.chunks = (int)hq_mx4_chunks(p->K, GROUP == BY_CHUNKS ? p->experts : 1);
    a.rows = p->K;
    a.outputs = outputs_of(p, GROUP);
    a.splits = plan.splits;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (plan.splits > 1) {
        if (!ws || ws_bytes < 4 * a.outputs * plan.splits || misaligned(ws, 16)) return HQ_E_WORKSPACE;
        a.out = ws;
        a.out_type = HQ_FP32;
    }
    if constexpr (GROUP != BY_CHUNKS) {
        if (plan.side <= 2) {
            a.n_tiles = tiles_of(p->N, 16);
            const long blocks = (long)a.n_tiles * p->experts;
            if (blocks >= 0x7fffffffL) return HQ_E_BADSHAPE;
            int waves = 1;
            while (waves < 8 && waves < a.chunks) waves *= 2;
            return hq_mx4_launch((unsigned)blocks, 64 * waves, [&](unsigned first, unsigned count) {
                a.first = first;
                if (plan.side == 2) hipLaunchKernelGGL((mx4_row_kernel<2, GROUP>), dim3(count), dim3(64 * waves), 0, s, a);
                else                hipLaunchKernelGGL((mx4_row_kernel<1, GROUP>), dim3(count), dim3(64 * waves), 0, s, a);
            });
        }
    }
    const int side = plan.side;
    const int used = std::min(p->experts, p->M);
    a.m_tiles = GROUP == BY_ROWS ? (p->M - used) / side + used : tiles_of(p->M, side);
    a.n_tiles = tiles_of(p->N, side);
    const double blocks = (double)a.m_tiles * a.n_tiles * (GROUP == BY_CHUNKS ? p->experts : 1) * a.splits;
    if (blocks >= 2147483648.0) return HQ_E_BADSHAPE;
    rc = side == 256 ? launch_tile<256, 256, 4, 2, GROUP>(a, (unsigned)blocks, s)
       : side == 128 ? launch_tile<128, 128, 2, 2, GROUP>(a, (unsigned)blocks, s) : launch_tile<64, 64, 2, 1, GROUP>(a, (unsigned)blocks, s);
    if (rc != HQ_OK || a.splits == 1) return rc;
    const float *part = static_cast<const float *>(ws);
    switch (p->out_type) {
    case HQ_FP32: launch_join<HQ_FP32>(part, a.outputs, a.splits, out, s); break;
    case HQ_BF16: launch_join<HQ_BF16>(part, a.outputs, a.splits, out, s); break;
    default:      launch_join<HQ_FP16>(part, a.outputs, a.splits, out, s); break;
    }
    return launch_status();
}

} // namespace

extern "C" {

size_t hq_mx4_workspace_bytes(int32_t entry, const hq_mx4_problem *p)
{
    if (entry != HQ_ENTRY_MX4_GEMM && entry != HQ_ENTRY_MX4_WGRAD_GROUPED) return 0;
    const int group = entry == HQ_ENTRY_MX4_GEMM ? DENSE : BY_CHUNKS;
    if (check_product(p, group != DENSE) != HQ_OK || p->M == 0 || p->N == 0) return 0;
    const Plan plan = plan_of(p, group);
    return plan.splits > 1 ? 4 * outputs_of(p, group) * (size_t)plan.splits : 0;
}

int hq_mx4_gemm(const hq_mx4_problem *p, const uint8_t *A, const uint8_t *As, const uint8_t *B, const uint8_t *Bs, void *out, void *ws,
                size_t ws_bytes, void *stream)
{
    return product<DENSE>(p, A, As, B, Bs, nullptr, out, ws, ws_bytes, stream);
}

int hq_mx4_gemm_grouped(const hq_mx4_problem *p, const uint8_t *A, const uint8_t *As, const uint8_t *B, const uint8_t *Bs,
                        const int32_t *offs, void *out, void *stream)
{
    return product<BY_ROWS>(p, A, As, B, Bs, offs, out, nullptr, 0, stream);
}

int hq_mx4_wgrad_grouped(const hq_mx4_problem *p, const uint8_t *A, const uint8_t *As, const uint8_t *B, const uint8_t *Bs,
                         const int32_t *offs, void *out, void *ws, size_t ws_bytes, void *stream)
{
    return product<BY_CHUNKS>(p, A, As, B, Bs, offs, out, ws, ws_bytes, stream);
}

} // extern "C"
