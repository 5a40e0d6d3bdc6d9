// The product with microscaled weights, Y = X W^T, and its gradients dX = dY W, dW = dY^T X.
// Forward: the scaled matrix instruction multiplies the codes as they are stored, 16 x 16 x 128 at a time, with one
// power of two per row and 32 values on either side.  W's rows are the instruction's rows and X's its
// columns, so a lane ends with four consecutive outputs of one token.
// The instruction adds products in groups of 16, aligned to the group's largest power of two and cut 13 bits below it (found by
// feeding it single codes): a small product beside two large ones that cancel would be gone.  Products of E2M1 alone reach over
// fewer bits.  E4M3's do not, so its codes are multiplied in two parts, those of 2 and more (the top bit of the exponent is set)
// and those below, each of which reaches over 13 bits: from 2^(8 + 2) to the last bit of 2^1 * 2^-1, 2^-3, and from 2^(0 + 2) to 2^-9 * 2^-1.
// Groups and parts add in fp32, so nothing is cut but what an fp32 sum cuts, at twice the instructions.  (Both parts of random codes
// came out exact to the last bit, and sums of normal data in fp32 are off by 2e-8 of their size where they were by 4.5e-6 in one part.
// 4096 x 4096 x 11008 takes 255 us instead of 170, 512 x 4096 x 4096 19 instead of 15, one token 8.8 instead of 8.0.)
// Gradients: the sums run along the other axes, across the blocks of 32, so the operands take part as bf16 (which holds
// code * 2^E exactly), transposed into scratch first, and both gradients are products of that same form.
#include "pv_ops.h"

namespace {

typedef int i8v __attribute__((ext_vector_type(8)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef pv_bf16 b8v __attribute__((ext_vector_type(8)));
typedef pv_bf16 b4v __attribute__((ext_vector_type(4)));

enum { kE2M1 = PV_MX_E2M1, kE4M3 = PV_MX_E4M3, kBF16 = 2 };

// an operand: rows of `pitch` bytes, nblk blocks of 32 values each
struct operand {
    const uint8_t *codes, *scales;      // scales: not for bf16
    int64_t pitch;
    int rows;
};

// Bytes of 128 values of a row, and where a lane's part of them lies: lane group q = lane / 16 holds values
// 32 q .. 32 q + 31 of E2M1, but 16 q .. + 15 and 64 + 16 q .. + 15 of E4M3; its scale is that of block q in either
// case.
template <int KIND>
struct part {
    static constexpr int chunks = KIND == kE2M1 ? 1 : 2;      // of 16 bytes, 4 lane groups each
    pv_u4 c[chunks];
    unsigned scale;
};

template <int KIND>
__device__ __forceinline__ void load_part(part<KIND> &p, const uint8_t *row, int step, int q, int nblk)
{
#pragma unroll
    for (int j = 0; j < part<KIND>::chunks; ++j) {
        // the chunk's place among the row's 16-byte pieces, and the block of 32 values that it belongs to
        const int piece = (step * part<KIND>::chunks + j) * 4 + q;
        const int block = KIND == kE2M1 ? piece : piece >> 1;
        p.c[j] = pv_u4{0u, 0u, 0u, 0u};
        if (block < nblk) p.c[j] = *reinterpret_cast<const pv_u4 *>(row + (int64_t)piece * 16);
    }
}

// scale bytes of the blocks of four steps, this lane group's block of each in the low byte; behind the row's end: 0
__device__ __forceinline__ pv_u4 load_scales(const uint8_t *scale_row, int step, int q, int nblk)
{
    typedef pv_u4 loose __attribute__((aligned(1)));
    pv_u4 v = {0u, 0u, 0u, 0u};
    if (step * 4 + 16 <= nblk) {
        v = *reinterpret_cast<const loose *>(scale_row + step * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = v[i] >> (8 * q) & 255u;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((step + i) * 4 + q < nblk) v[i] = scale_row[(step + i) * 4 + q];
    }
    return v;
}

// Four codes of E4M3 in two parts: the codes whose bit 6 is set (`low` becomes the others, in their places).  A byte's selector
// above 12 selects 0xff, and 0 the source's lowest byte, here a zero.
__device__ __forceinline__ unsigned upper_codes(unsigned &low)
{
    const unsigned upper = low & __builtin_amdgcn_perm(0u, 0u, low & 0x40404040u);
    low ^= upper;
    return upper;
}

template <int WK, int XK>
__device__ __forceinline__ f4v multiply(const part<WK> &w, const part<XK> &x, f4v acc)
{
    constexpr int kA = WK == kE2M1 ? 4 : 0, kB = XK == kE2M1 ? 4 : 0;
    i8v a = {0, 0, 0, 0, 0, 0, 0, 0}, b = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < part<WK>::chunks * 4; ++i) a[i] = (int)w.c[i / 4][i % 4];
#pragma unroll
    for (int i = 0; i < part<XK>::chunks * 4; ++i) b[i] = (int)x.c[i / 4][i % 4];
    if constexpr (XK == kE4M3) {
        i8v upper;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            unsigned low = (unsigned)b[i];
            upper[i] = (int)upper_codes(low);
            b[i] = (int)low;
        }
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, upper, acc, kA, kB, 0, (int)w.scale, 0, (int)x.scale);
    }
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, kA, kB, 0, (int)w.scale, 0, (int)x.scale);
}

// four consecutive outputs of one row of Y
template <class T>
__device__ __forceinline__ void store_four(T *y, int left, bool whole, f4v v)
{
    if (whole) {
        typedef T four __attribute__((ext_vector_type(4)));
        *reinterpret_cast<four *>(y) = four{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) y[i] = (T)v[i];
}

// Few tokens: 16 rows of W and 16 of X a block, straight from memory to registers.  Bound by W's bytes and by the way there: the
// waves take four steps of 128 values each in turn, ask for all of them before they multiply the first, and meet in LDS.
// Eight waves where there are no more than two blocks a compute unit, else four (1 token, us with 4 | 8 waves: 4096 -> 11008
// 8.8 | 9.1, 14336 -> 4096 14.6 | 10.8; 24 and 31 MB of W, where a launch that does next to nothing takes 3).
constexpr int kBatch = 4;

template <int WK, int XK, int WAVES, class T>
__global__ __launch_bounds__(WAVES * 64) void k_product_direct(operand w, operand x, int nblk, T *__restrict__ Y, int wtiles)
{
    __shared__ f4v sums[WAVES - 1][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4, r = lane & 15;
    const int o0 = blockIdx.x % wtiles * 16, t0 = blockIdx.x / wtiles * 16;
    const int steps = (nblk + 3) / 4;
    // rows past the end repeat the last one; their results are not stored
    const int wrow = min(o0 + r, w.rows - 1), xrow = min(t0 + r, x.rows - 1);
    const uint8_t *wp = w.codes + wrow * w.pitch, *ws = w.scales + (int64_t)wrow * nblk;
    const uint8_t *xp = x.codes + xrow * x.pitch, *xs = x.scales + (int64_t)xrow * nblk;
    f4v acc = {0.0f, 0.0f, 0.0f, 0.0f};
    static_assert(kBatch == 4, "as many steps as load_scales brings");
    for (int s = wave * kBatch; s < steps; s += WAVES * kBatch) {
        part<WK> a[kBatch];
        part<XK> b[kBatch];
        const pv_u4 as = load_scales(ws, s, q, nblk), bs = load_scales(xs, s, q, nblk);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {           // behind the last step: zeros
            load_part(a[i], wp, s + i, q, nblk);
            load_part(b[i], xp, s + i, q, nblk);
            a[i].scale = as[i];
            b[i].scale = bs[i];
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) acc = multiply(a[i], b[i], acc);
    }
    // the last instructions run here, by every lane, not inside a branch that stores their results
    asm volatile("" : "+v"(acc));
    if (wave) sums[wave - 1][lane] = acc;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 0; i < WAVES - 1; ++i) acc += sums[i][lane];
    const int t = t0 + r, o = o0 + q * 4;
    if (t < x.rows && o < w.rows) store_four(Y + (int64_t)t * w.rows + o, w.rows - o, (w.rows & 3) == 0, acc);
}

// ---------------------------------------------------------------- tiles through LDS

// A step is 128 values of a microscaled row or 64 of a bf16 one: `bytes` of it, in pieces of 16.  It is multiplied in slices, one
// instruction's depth each: 32 x 32 x 64 on codes, 32 x 32 x 16 on bf16.
template <int KIND>
struct step_of {
    static constexpr int bytes = KIND == kE2M1 ? 64 : 128, pieces = bytes / 16;
    static constexpr int values = KIND == kBF16 ? 64 : 128, blocks = values / 32;
    static constexpr int slices = KIND == kBF16 ? 4 : 2;
};

// Where piece c of a tile's row lies in LDS: rows are `bytes` apart, and the pieces of a row change places by a key
// of the row, so that lanes which read the same piece of neighbouring rows meet different banks.
template <int KIND>
__device__ __forceinline__ int key_of(int row)
{
    if constexpr (step_of<KIND>::pieces == 8) return (row & 3) | (row >> 3 & 1) << 2;
    return (row >> 1 & 1) | (row >> 3 & 1) << 1;
}

// A lane's part of 32 rows of a slice: 32 values of codes (lane group h = lane / 32: block h; E4M3 in two halves of 16 values, 16 h
// and 32 + 16 h), or 8 values of bf16, 8 h.
template <int KIND>
struct frag {
    pv_u4 c[KIND == kE4M3 ? 2 : 1];
};

template <int KIND>
__device__ __forceinline__ int piece_in_step(int slice, int c, int h)
{
    return KIND == kE4M3 ? slice * 4 + c * 2 + h : slice * 2 + h;
}

// the part of a fragment's codes that is multiplied by itself; the fragment keeps the others
template <int KIND>
__device__ __forceinline__ frag<KIND> upper_part(frag<KIND> &f)
{
    frag<KIND> u = f;
    if constexpr (KIND == kE4M3) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unsigned low = f.c[c][i];
                u.c[c][i] = upper_codes(low);
                f.c[c][i] = low;
            }
    }
    return u;
}

// ws, xs: the scales of the step's blocks h and 2 + h in bytes 0 and 2; SEL: the slice's byte
template <int SEL, int WK, int XK>
__device__ __forceinline__ f16v multiply(const frag<WK> &w, unsigned ws, const frag<XK> &x, unsigned xs, f16v acc)
{
    if constexpr (WK == kBF16) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8v, w.c[0]), __builtin_bit_cast(b8v, x.c[0]), acc, 0, 0, 0);
    } else {
        i8v a = {0, 0, 0, 0, 0, 0, 0, 0}, b = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = (int)w.c[0][i];
#pragma unroll
        for (int i = 0; i < (XK == kE4M3 ? 8 : 4); ++i) b[i] = (int)x.c[i / 4][i % 4];
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 4, XK == kE2M1 ? 4 : 0, SEL, (int)ws, SEL, (int)xs);
    }
}

// BYTES (16 or 4) a lane from memory, `far` behind a scalar address, to LDS, lane i to `to` + BYTES * i.  An instruction and no
// builtin: behind the builtin the compiler takes every later read of LDS for one that may be answered out of order, and waits for
// all of them at each use (4096 x 8192 x 4096: 113 -> 107 us).  It has no result; the kernel waits for it by count.  It reads m0 one
// wait state after a scalar instruction has written it at the earliest, and its address five after a vector instruction; the compiler,
// which counts those for its own instructions, does not look in here.  (The address comes from scalar instructions alone.)
template <int BYTES>
__device__ __forceinline__ void fetch(const void *from, unsigned far, unsigned to)
{
    if constexpr (BYTES == 16) asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(far), "s"(from), "{m0}"(to) : "memory");
    else asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(far), "s"(from), "{m0}"(to) : "memory");
}

// All but the last N memory operations of this wave are done, its reads of LDS too, and every wave has come here.
template <int N>
__device__ __forceinline__ void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

struct tiling {
    int nblk;                // blocks of 32 values a row
    int wtiles, xtiles;
    int splits;              // of the steps
    int64_t scale_pitch;     // bytes, a multiple of 4 (microscaled)
    float *partial;          // splits > 1: [splits][x.rows][w.rows]
};

// BM rows of W times BN rows of X a block of WM x WN waves, NS stages of a step each in LDS.
// The matrix cores wait for nothing that can be asked for earlier: while a slice is multiplied, the next one is read from LDS into
// a second set of registers, the first of the next step behind the last of this one.  So the waves meet before a step's last
// slice: then all have this step in registers, its stage is free for the loads of step s + NS, and step s + 1 has arrived.
// Rows of W are dealt to the instruction's rows so that a lane ends with eight consecutive outputs of a token: its row
// 16 a + 8 b + 4 c + i (b, c bits, i < 4) is row 16 a + 8 c + 4 b + i.
template <int WK, int XK, int BM, int BN, int WM, int WN, int NS, class T>
__global__ __launch_bounds__(WM *WN * 64) void k_product_tiled(operand w, operand x, tiling p, T *__restrict__ Y)
{
    constexpr int kWaves = WM * WN, kThreads = kWaves * 64, FM = BM / WM / 32, FN = BN / WN / 32;
    constexpr int kWBytes = BM * step_of<WK>::bytes, kXBytes = BN * step_of<XK>::bytes;
    // scales: four steps of them at a time, 16 bytes a row, in two buffers behind the stages
    constexpr int kScales = WK == kBF16 ? 0 : (BM + BN) * 16;
    constexpr int kStage = kWBytes + kXBytes;
    constexpr int kWLoads = kWBytes / 1024 / kWaves, kXLoads = kXBytes / 1024 / kWaves, kData = kWLoads + kXLoads;
    constexpr int kSLoads = WK == kBF16 ? 0 : (BM + BN + 64 * kWaves - 1) / 64 / kWaves;
    constexpr int kSlices = step_of<WK>::slices;
    // instructions stay where they are written, but for the narrow tile's parts of E4M3, which have nothing else to run beside
    // (512 tokens, 4096 -> 4096: 19.5 -> 18.8 us)
    constexpr bool kFenced = XK != kE4M3 || FN > 1;
    static_assert(kWLoads * 1024 * kWaves == kWBytes && kXLoads * 1024 * kWaves == kXBytes, "whole loads a wave");
    static_assert(BM % 16 == 0 && FM * 32 * WM == BM && FN * 32 * WN == BN && kSlices % 2 == 0 && NS >= 2, "tile");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[NS * kStage + 2 * kScales];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane >> 5, r = lane & 31;
    // blocks are dealt to the eight dies in turn: each die gets a stretch of the tiles, and walks it in bands of four tiles
    // of X, so that what its blocks read together stays in its L2
    const int tiles = p.wtiles * p.xtiles, split = blockIdx.x / tiles;
    int tile = blockIdx.x - split * tiles;
    {
        const int die = tile & 7, per = tiles >> 3, extra = tiles & 7;
        tile = die * per + min(die, extra) + (tile >> 3);
    }
    const int band = tile / (4 * p.wtiles), in_band = tile - band * 4 * p.wtiles, deep = min(4, p.xtiles - band * 4);
    const int wt = in_band / deep, xt = band * 4 + in_band - wt * deep;
    const int o0 = wt * BM, t0 = xt * BN;

    const int all = (p.nblk + step_of<WK>::blocks - 1) / step_of<WK>::blocks;
    const int s0 = (int)((int64_t)all * split / p.splits), s1 = (int)((int64_t)all * (split + 1) / p.splits);
    const bool tail = s1 == all && p.nblk % step_of<WK>::blocks != 0;      // the last step is part of one
    const int steps = s1 - s0, whole = steps - (tail ? 1 : 0);

    const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    // Sources of this wave's loads of a step: a scalar address that moves with the steps, and a lane's 32-bit distance from it.
    // Rows past the end repeat the last one, their results are not stored.
    const uint8_t *wsrc = w.codes + (int64_t)o0 * w.pitch + (int64_t)s0 * step_of<WK>::bytes;
    const uint8_t *xsrc = x.codes + (int64_t)t0 * x.pitch + (int64_t)s0 * step_of<XK>::bytes;
    unsigned far[kData];
#pragma unroll
    for (int i = 0; i < kWLoads; ++i) {
        const int at = (i * kWaves + wave) * 64 + lane, row = at / step_of<WK>::pieces, c = at % step_of<WK>::pieces;
        far[i] = (unsigned)min(row, w.rows - 1 - o0) * (unsigned)w.pitch + (c ^ key_of<WK>(row)) * 16;
    }
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) {
        const int at = (i * kWaves + wave) * 64 + lane, row = at / step_of<XK>::pieces, c = at % step_of<XK>::pieces;
        far[kWLoads + i] = (unsigned)min(row, x.rows - 1 - t0) * (unsigned)x.pitch + (c ^ key_of<XK>(row)) * 16;
    }
    // loads `first` .. `last` - 1 of the next step that has not been asked for, into `stage`
    auto fetch_some = [&](int stage, int first, int last) {
        const unsigned to = base + stage * kStage + wave * 1024;
#pragma unroll
        for (int i = 0; i < kData; ++i) {
            if (i < first || i >= last) continue;
            if (i < kWLoads) fetch<16>(wsrc, far[i], to + i * kWaves * 1024);
            else fetch<16>(xsrc, far[i], to + kWBytes + (i - kWLoads) * kWaves * 1024);
        }
        if (last == kData) {
            wsrc += step_of<WK>::bytes;
            xsrc += step_of<XK>::bytes;
        }
    };
    auto fetch_step = [&](int stage) { fetch_some(stage, 0, kData); };
    // A load of scales: 16 rows, four steps of one row side by side, so that a line of memory is asked for once in four steps.
    // What lies behind the row's end is not used and stands for the last blocks.
    const int wlast = w.rows - 1 - o0, xlast = x.rows - 1 - t0, last_scales = ((p.nblk - 1) & ~3) - s0 * 4;
    const uint8_t *wscale = w.scales + (int64_t)o0 * p.scale_pitch + (int64_t)s0 * 4, *xscale = x.scales + (int64_t)t0 * p.scale_pitch + (int64_t)s0 * 4;
    auto fetch_scales = [&](int quarter, int group) {
        if (WK == kBF16) return;
        const unsigned at = (unsigned)min((group * 4 + (lane & 3)) * 4, last_scales);
#pragma unroll
        for (int i = 0; i < kSLoads; ++i) {
            const int first = ((quarter * kSLoads + i) * kWaves + wave) * 16;
            if (first >= BM + BN) continue;
            const bool of_w = first < BM;
            const int row = min((of_w ? first : first - BM) + (lane >> 2), of_w ? wlast : xlast);
            fetch<4>(of_w ? wscale : xscale, (unsigned)row * (unsigned)p.scale_pitch + at, base + NS * kStage + (group & 1) * kScales + first * 16);
        }
    };
    // The step that is part of one: through registers, with zeros behind the row's last block.
    auto copy_tail = [&](int stage) {
        const int b0 = (s1 - 1) * step_of<WK>::blocks;
        auto copy = [&](auto kind, const operand &o, int first, int rows, unsigned at) {
            constexpr int KIND = decltype(kind)::value, kPieces = step_of<KIND>::pieces, kPerBlock = kPieces / step_of<KIND>::blocks;
            for (int i = threadIdx.x; i < rows * kPieces; i += kThreads) {
                const int row = i / kPieces, c = i % kPieces;
                pv_u4 v = {0u, 0u, 0u, 0u};
                if (b0 + c / kPerBlock < p.nblk)
                    v = *reinterpret_cast<const pv_u4 *>(o.codes + (int64_t)min(first + row, o.rows - 1) * o.pitch + (int64_t)(s1 - 1) * step_of<KIND>::bytes + c * 16);
                *reinterpret_cast<pv_u4 *>(lds + stage * kStage + at + row * step_of<KIND>::bytes + (c ^ key_of<KIND>(row)) * 16) = v;
            }
        };
        copy(std::integral_constant<int, WK>{}, w, o0, BM, 0);
        copy(std::integral_constant<int, XK>{}, x, t0, BN, kWBytes);
    };

    // this lane's rows of the first fragments
    const int wr = (wave / WN) * (BM / WM) + ((r & 19) | (r >> 2 & 1) << 3 | (r >> 3 & 1) << 2), xr = (wave % WN) * (BN / WN) + r;
    frag<WK> a[FM];
    frag<XK> b[2][FN];
    unsigned ws[FM], xs[FN], xs_next[FN];      // scales as they come, four blocks a row; of the step at hand moved to this lane's blocks
    auto read_x = [&](int set, int stage, int step, int slice) {
        const uint8_t *xl = lds + stage * kStage + kWBytes + xr * step_of<XK>::bytes;
        const uint8_t *sc = lds + NS * kStage + (step >> 2 & 1) * kScales + (step & 3) * 4;
#pragma unroll
        for (int n = 0; n < FN; ++n) {
#pragma unroll
            for (int c = 0; c < (XK == kE4M3 ? 2 : 1); ++c)
                b[set][n].c[c] = *reinterpret_cast<const pv_u4 *>(xl + n * 32 * step_of<XK>::bytes + (piece_in_step<XK>(slice, c, h) ^ key_of<XK>(xr)) * 16);
            if (WK != kBF16 && slice == 0) xs_next[n] = *reinterpret_cast<const unsigned *>(sc + (BM + xr + n * 32) * 16);
        }
    };
    auto read_w = [&](int m, int stage, int step, int slice) {
        const uint8_t *wl = lds + stage * kStage + wr * step_of<WK>::bytes;
        const uint8_t *sc = lds + NS * kStage + (step >> 2 & 1) * kScales + (step & 3) * 4;
        a[m].c[0] = *reinterpret_cast<const pv_u4 *>(wl + m * 32 * step_of<WK>::bytes + (piece_in_step<WK>(slice, 0, h) ^ key_of<WK>(wr)) * 16);
        if (WK != kBF16 && slice == 0) ws[m] = *reinterpret_cast<const unsigned *>(sc + (wr + m * 32) * 16);
    };
    // X in E4M3 is multiplied in two parts: of the first fragment they are formed while the slice before is multiplied, of the others
    // behind the slice's first instructions
    frag<XK> upper[FN == 1 ? 2 : 1][FN];
    f16v acc[FM][FN];
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n = 0; n < FN; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.0f;

#pragma unroll
    for (int i = 0; i < 4; ++i) fetch_scales(i, 0);
    if (steps > 4) fetch_scales(0, 1);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        if (s < whole) fetch_step(s);
        else if (s == whole && tail) copy_tail(s);
    }
    if (NS <= whole) wait_and_meet<(NS - 1) * kData>();
    else wait_and_meet<0>();
    read_x(0, 0, 0, 0);
#pragma unroll
    for (int m = 0; m < FM; ++m) read_w(m, 0, 0, 0);
    if constexpr (XK == kE4M3) upper[0][0] = upper_part(b[0][0]);
    // Loads that may be on their way when step s + 1 has to have arrived: those of the steps s + 2 .. s + NS - 1; of scales, the last
    // ones that are needed were asked for right before the last of those steps.
    constexpr int kAhead = (WK == kBF16 ? NS - 2 : NS > 2 ? 1 : 0) * kData;
    int stage = 0;
    // A step.  FULL: there is a whole step s + NS, and no condition stands between the instructions.  What is read behind the last
    // step is not used.
    auto step = [&](auto full, int s) {
        constexpr bool FULL = decltype(full)::value;
        const int after = stage + 1 == NS ? 0 : stage + 1;
#pragma unroll
        for (int j = 0; j < kSlices; ++j) {
            const bool last = j + 1 == kSlices;
            const int to_stage = last ? after : stage, to_step = last ? s + 1 : s, to_slice = last ? 0 : j + 1;
            if (!last) read_x((j + 1) & 1, to_stage, to_step, to_slice);
            const int set = j & 1, mine = FN == 1 ? set : 0, its = FN == 1 ? set ^ 1 : 0;
            // a fragment of W's rows is read over as soon as its instructions have taken it
#pragma unroll
            for (int m = 0; m < FM; ++m) {
                if constexpr (kFenced) __builtin_amdgcn_sched_barrier(0);
                if (j == 0 && WK != kBF16) {
                    ws[m] >>= 8 * h;
#pragma unroll
                    for (int n = 0; n < FN; ++n)
                        if (m == 0) xs[n] = xs_next[n] >> (8 * h);
                }
#pragma unroll
                for (int n = 0; n < FN; ++n) {
                    auto add = [&](const frag<XK> &x) {
                        acc[m][n] = j & 1 ? multiply<2>(a[m], ws[m], x, xs[n], acc[m][n]) : multiply<0>(a[m], ws[m], x, xs[n], acc[m][n]);
                    };
                    if constexpr (XK == kE4M3) {
                        if (n > 0 && m == 0) upper[0][n] = upper_part(b[set][n]);
                        add(upper[mine][n]);
                    }
                    add(b[set][n]);
                    if (XK == kE4M3 && n == 0 && m == FM - 1) upper[its][0] = upper_part(b[set ^ 1][0]);
                }
                if constexpr (kFenced) __builtin_amdgcn_sched_barrier(0);
                if (last && m == 0) {
                    if constexpr (FULL) {
                        wait_and_meet<kAhead>();
                        fetch_scales((s + 1) & 3, ((s + 1) >> 2) + 1);
                    } else {
                        wait_and_meet<0>();
                        if ((((s + 1) >> 2) + 1) * 4 < steps) fetch_scales((s + 1) & 3, ((s + 1) >> 2) + 1);
                        if (s + NS == whole && tail) copy_tail(stage);
                    }
                    read_x(0, to_stage, to_step, to_slice);
                }
                if (FULL && last) fetch_some(stage, m * kData / FM, (m + 1) * kData / FM);
                read_w(m, to_stage, to_step, to_slice);
            }
        }
        stage = after;
    };
    __builtin_amdgcn_s_waitcnt(0xC07F);        // lgkmcnt(0), seen by the compiler: no scalar load is left that its count would have to allow for
    int s = 0;
    for (; s + NS < whole; ++s) step(std::true_type{}, s);
    for (; s < steps; ++s) step(std::false_type{}, s);
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            // every lane runs the last instructions, whatever it stores
            asm volatile("" : "+v"(acc[m][n]));
            const int t = t0 + xr + n * 32;
            if (t >= x.rows) continue;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int o = o0 + (wave / WN) * (BM / WM) + m * 32 + e * 16 + h * 8;
                if (o >= w.rows) continue;
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = acc[m][n][e * 8 + i];
                if (p.splits == 1) pv_store8(Y + (int64_t)t * w.rows + o, w.rows - o, v);
                else pv_store8(p.partial + ((int64_t)split * x.rows + t) * w.rows + o, w.rows - o, v);
            }
        }
}

// the splits' sums added in their order
template <class T>
__global__ __launch_bounds__(256) void k_add_splits(const float *__restrict__ partial, int splits, int64_t n, T *__restrict__ Y)
{
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= n) return;
    const int valid = (int)min(n - at, (int64_t)8);
    float v[8];
    pv_load8(partial + at, valid, v);
    for (int s = 1; s < splits; ++s) {
        float u[8];
        pv_load8(partial + s * n + at, valid, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += u[i];
    }
    pv_store8(Y + at, valid, v);
}

// scales with rows of a pitch that is a multiple of 4, zeros behind
__global__ __launch_bounds__(256) void k_pad_scales(const uint8_t *__restrict__ in, int64_t rows, int nblk, uint8_t *__restrict__ out, int pitch)
{
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, per = pitch / 4, row = u / per;
    if (row >= rows) return;
    const int c = (int)(u - row * per) * 4;
    unsigned v = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) v |= (c + i < nblk ? (unsigned)in[row * nblk + c + i] : 0u) << (8 * i);
    reinterpret_cast<unsigned *>(out)[u] = v;
}

// ---------------------------------------------------------------- operands of the gradients

// A matrix [rows, cols] (codes, or bf16) as bf16, transposed: out [cols, pitch] with pitch >= rows, zeros behind `rows`.
struct turned {
    const uint8_t *codes, *scales;
    pv_bf16 *out;
    int64_t rows, cols, pitch;
    int kind, nblk;
    unsigned ctiles, blocks;
};

// 16 consecutive values of a row as eight words of bf16 pairs; zeros outside the matrix
template <int KIND>
__device__ __forceinline__ void load_pairs(const turned &m, int64_t row, int64_t col, unsigned (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0u;
    if (row >= m.rows) return;
    if constexpr (KIND == kBF16) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int64_t at = col + 8 * half;
            const b8v r = pv_load8_raw(reinterpret_cast<const pv_bf16 *>(m.codes) + row * m.cols + at, (int)max(min(m.cols - at, (int64_t)8), (int64_t)0));
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * half + i] = __builtin_bit_cast(pv_u4, r)[i];
        }
    } else {
        if (col >= (int64_t)m.nblk * kMxBlock) return;
        const float power = pv_mx_power(m.scales[row * m.nblk + col / kMxBlock]);
        const int64_t at = row * m.nblk * (KIND == kE2M1 ? 16 : 32) + (KIND == kE2M1 ? col / 2 : col);
        if constexpr (KIND == kE2M1) {
            const pv_u2 c = *reinterpret_cast<const pv_u2 *>(m.codes + at);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                v[4 * i + 0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], power, 0));
                v[4 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], power, 1));
                v[4 * i + 2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], power, 2));
                v[4 * i + 3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], power, 3));
            }
        } else {
            const pv_u4 c = *reinterpret_cast<const pv_u4 *>(m.codes + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i + 0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], power, false));
                v[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[i], power, true));
            }
        }
    }
}

// Up to three matrices in one launch, in tiles of 64 x 64 through LDS.  Rows there are 33 words apart: the 64 lanes that read a
// word each - 8 pairs of columns of 8 rows 8 apart - meet 64 banks.  Bound by the bytes, most of them written.
__global__ __launch_bounds__(256) void k_transpose(turned m0, turned m1, turned m2)
{
    __shared__ unsigned tile[64][33];
    unsigned b = blockIdx.x;
    const bool first = b < m0.blocks, second = !first && b - m0.blocks < m1.blocks;
    const turned m = first ? m0 : second ? m1 : m2;
    b -= first ? 0 : second ? m0.blocks : m0.blocks + m1.blocks;
    const int64_t r0 = (int64_t)(b / m.ctiles) * 64, c0 = (int64_t)(b % m.ctiles) * 64;
    {
        const int r = threadIdx.x >> 2, c = (threadIdx.x & 3) * 16;
        unsigned v[8];
        if (m.kind == kE2M1) load_pairs<kE2M1>(m, r0 + r, c0 + c, v);
        else if (m.kind == kE4M3) load_pairs<kE4M3>(m, r0 + r, c0 + c, v);
        else load_pairs<kBF16>(m, r0 + r, c0 + c, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) tile[r][c / 2 + i] = v[i];
    }
    __syncthreads();
    const int c = threadIdx.x >> 3, r = (threadIdx.x & 7) * 8;
    unsigned v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = tile[r + i][c];
    if (r0 + r >= m.pitch) return;                     // (a multiple of 8)
#pragma unroll
    for (int odd = 0; odd < 2; ++odd) {
        const int64_t col = c0 + 2 * c + odd;
        if (col >= m.cols) return;
        pv_u4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], odd ? 0x07060302u : 0x05040100u);
        *reinterpret_cast<pv_u4 *>(m.out + col * m.pitch + r0 + r) = o;
    }
}

// bf16 rows of `cols` to rows of `pitch`, zeros behind
__global__ __launch_bounds__(256) void k_pad_rows(const pv_bf16 *__restrict__ in, int64_t rows, int64_t cols,
                                                  pv_bf16 *__restrict__ out, int64_t pitch)
{
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, per = pitch / 8;
    const int64_t row = u / per, col = (u - row * per) * 8;
    if (row >= rows) return;
    float v[8];
    pv_load8(in + row * cols + col, (int)min(cols - col, (int64_t)8), v);
    pv_store8(out + row * pitch + col, 8, v);
}

// ---------------------------------------------------------------- which kernel

// tiles of W's rows by X's: 128 x 64, 128 x 128 (both two blocks a compute unit) and 256 x 256 (one)
constexpr int kNarrow = 0, kMiddle = 1, kLarge = 2, kDirect = 3;

struct choice {
    int tile, splits;
    size_t partial;          // bytes of the splits' sums
};

// The variant that is expected to take least, from what the parts take: a step of one block or of two on a compute unit, in parts of
// a large tile's step (us); a launch's start and end; another launch that adds the splits' sums, which are written and read.
// Measured (us), 4096 -> 4096, e4m3, bf16 out, narrow | middle | large tiles, with 1, 2, 4 splits:
//   64 tokens 17.8 14.3 12.4 | 29.9 20.3 15.3        128 tokens 18.0 15.3 14.7 | 30.0 22.2 18.3 | 74.0 45.3 31.0
//   300 tokens 18.3 22.7 24.4 | 30.1 25.5 26.0         without splits: 512 tokens 19.1 | 30.5 | 75.2, 1024 tokens 30.9 | 32.9 | 76.3,
//   2048 tokens 62.8 | 56.3 | 82.9, 3000 tokens 87.5 | 80.2 | 83.8, 4096 tokens 110 | 103 | 89
//   131 tokens 14336 -> 4096, both e2m1, f32 out, with 1, 2, 4, 8: 36.2 24.0 22.3 23.4 | 45.6 29.4 21.6 24.6
// Up to 16 tokens W is read straight to registers, at any size (32 tokens, 4096 -> 11008: 21.0 that way, 14.6 through tiles).
template <int WK, int XK>
choice choose(int64_t out, int64_t tokens, int nblk)
{
    constexpr struct {
        int bm, bn, at_once;
        double one, two;
    } kTiles[] = {{128, 64, 512, 0.175, XK == kE4M3 ? 0.335 : 0.375}, {128, 128, 512, WK == kBF16 ? 0.4 : XK == kE4M3 ? 0.32 : 0.28, XK == kE4M3 ? 0.65 : 0.6}, {256, 256, 256, 1.0, 1.0}};
    constexpr double kStep = WK == kBF16 ? 1.5 : XK == kE4M3 ? 2.5 : 1.15;
    const int steps = (nblk + step_of<WK>::blocks - 1) / step_of<WK>::blocks;
    choice best = {kLarge, 1, 0};
    double least = 1e300;
    for (int tile = kNarrow; tile <= kLarge; ++tile) {
        const auto &t = kTiles[tile];
        const int64_t tiles = ((out + t.bm - 1) / t.bm) * ((tokens + t.bn - 1) / t.bn);
        for (int splits = 1; splits <= 16 && splits * 4 <= (steps > 4 ? steps : 4); splits *= 2) {
            const int64_t blocks = tiles * splits, rounds = blocks / t.at_once, rest = blocks % t.at_once;
            const double mine = (double)((steps + splits - 1) / splits) * kStep;
            double us = (double)rounds * (mine * t.two + 4.0);
            if (rest) us += mine * (rest <= 256 ? t.one : t.two) + 4.0;
            if (splits > 1) us += 4.0 + (double)splits * (double)(out * tokens) * 8 / 4e6;
            if (us < least) least = us, best = {tile, splits, splits > 1 ? (size_t)(splits * out * tokens) * 4 : 0};
        }
    }
    return best;
}

template <int WK, int XK, int BM, int BN, int WM, int WN, int NS, class T>
pv_status launch_tiled(pv_ctx *ctx, const operand &w, const operand &x, tiling p, T *Y)
{
    p.wtiles = (w.rows + BM - 1) / BM;
    p.xtiles = (x.rows + BN - 1) / BN;
    const int64_t blocks = (int64_t)p.wtiles * p.xtiles * p.splits;
    if (!pv_grid_fits(blocks, WM * WN * 64)) return pv_fail(ctx, PV_ERR_UNSUPPORTED, "too many tiles of the product");
    hipLaunchKernelGGL((k_product_tiled<WK, XK, BM, BN, WM, WN, NS, T>), dim3((unsigned)blocks), dim3(WM * WN * 64), 0, ctx->stream, w, x, p, Y);
    PV_HIP(ctx, hipGetLastError());
    if (p.splits == 1) return PV_OK;
    const int64_t n = (int64_t)x.rows * w.rows, sums = (n + 2047) / 2048;
    if (!pv_grid_fits(sums, 256)) return pv_fail(ctx, PV_ERR_UNSUPPORTED, "too many outputs of the product");
    hipLaunchKernelGGL((k_add_splits<T>), dim3((unsigned)sums), dim3(256), 0, ctx->stream, p.partial, p.splits, n, Y);
    PV_HIP(ctx, hipGetLastError());
    return PV_OK;
}

template <int WK, int XK, class T>
pv_status launch_direct(pv_ctx *ctx, const operand &w, const operand &x, int nblk, T *Y)
{
    const int wtiles = (w.rows + 15) / 16;
    const int64_t blocks = (int64_t)wtiles * ((x.rows + 15) / 16);
    if (!pv_grid_fits(blocks, 256)) return pv_fail(ctx, PV_ERR_UNSUPPORTED, "too many tiles of the product");
    const bool few = blocks <= 512;
    const auto k = few ? k_product_direct<WK, XK, 8, T> : k_product_direct<WK, XK, 4, T>;
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(few ? 512 : 256), 0, ctx->stream, w, x, nblk, Y, wtiles);
    PV_HIP(ctx, hipGetLastError());
    return PV_OK;
}

// w, x: with scale rows of `scale_pitch` bytes, a multiple of 4; partial: room for the splits' sums
template <int WK, int XK, class T>
pv_status launch(pv_ctx *ctx, const choice &c, const operand &w, const operand &x, int nblk, int64_t scale_pitch, float *partial, T *Y)
{
    const tiling p = {nblk, 0, 0, c.splits, scale_pitch, partial};
    // Stages: as many as LDS holds for two blocks of the smaller tiles or one of the large, but no more than three.  (bf16, narrow,
    // gradients of 256 x 2048 x 1024: two 23.2 us, three 20.3; codes with four or five stages take what they take with three:
    // what the smaller tiles wait for is the rate of the L2, 15 TB/s of the 256 compute units together.)
    constexpr int NS = WK == kBF16 ? 2 : 3;
    if (c.tile == kNarrow) return launch_tiled<WK, XK, 128, 64, 2, 2, 3>(ctx, w, x, p, Y);
    if (c.tile == kMiddle) return launch_tiled<WK, XK, 128, 128, 2, 2, NS>(ctx, w, x, p, Y);
    return launch_tiled<WK, XK, 256, 256, 2, 4, NS>(ctx, w, x, p, Y);
}

operand coded(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, int format)
{
    return {codes, scales, pv_mx_blocks(cols) * (format == PV_MX_E2M1 ? 16 : 32), (int)rows};
}

operand plain(const void *p, int64_t rows, int64_t pitch) { return {static_cast<const uint8_t *>(p), nullptr, pitch * 2, (int)rows}; }

int64_t padded(int64_t n) { return pv_mx_blocks(n) * kMxBlock; }


size_t round16(size_t bytes) { return (bytes + 15) & ~(size_t)15; }

turned turn(int kind, const void *codes, const uint8_t *scales, int64_t rows, int64_t cols, pv_bf16 *out)
{
    const int64_t pitch = padded(rows), ctiles = (cols + 63) / 64, blocks = ctiles * ((pitch + 63) / 64);
    // (a side is below 2^31, and products of 2^25 tiles either way do not fit memory: what is too large shows as 2^31)
    return {static_cast<const uint8_t *>(codes), scales, out, rows, cols, pitch, kind, (int)pv_mx_blocks(cols), (unsigned)ctiles,
            (unsigned)(blocks < ((int64_t)1 << 31) ? blocks : (int64_t)1 << 31)};
}

pv_status transpose(pv_ctx *ctx, const turned *m, int n)
{
    const turned none = {};
    const int64_t blocks = (int64_t)m[0].blocks + (n > 1 ? m[1].blocks : 0) + (n > 2 ? m[2].blocks : 0);
    if (!pv_grid_fits(blocks, 256)) return pv_fail(ctx, PV_ERR_UNSUPPORTED, "too many tiles of the gradients' operands");
    hipLaunchKernelGGL(k_transpose, dim3((unsigned)blocks), dim3(256), 0, ctx->stream, m[0], n > 1 ? m[1] : none, n > 2 ? m[2] : none);
    PV_HIP(ctx, hipGetLastError());
    return PV_OK;
}

// A tile's rows lie within 32 bits of its first: a row of an operand is below 16 MiB.  Asked before anything is enqueued.
pv_status check_pitch(pv_ctx *ctx, int64_t bytes)
{
    if (bytes < 1 << 24) return PV_OK;
    return pv_fail(ctx, PV_ERR_UNSUPPORTED, "a row of %lld bytes of an operand: 16 MiB or more", (long long)bytes);
}

}  // namespace

pv_status pv_launch_mx_product(pv_ctx *ctx, int64_t tokens, int64_t out, int64_t in, int x_format,
                               const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *w_codes,
                               const uint8_t *w_scales, int y_type, void *Y)
{
    operand w = coded(w_codes, w_scales, out, in, PV_MX_E2M1), x = coded(x_codes, x_scales, tokens, in, x_format);
    const int nblk = (int)pv_mx_blocks(in);
    const choice c = tokens <= 16 ? choice{kDirect, 1, 0}
                   : x_format == PV_MX_E2M1 ? choose<kE2M1, kE2M1>(out, tokens, nblk) : choose<kE2M1, kE4M3>(out, tokens, nblk);
    if (c.tile == kDirect) {
        pv_timed t(ctx, PV_K_MX_PRODUCT);
        return pv_for_dtype(y_type, [&](auto v) {
            using T = decltype(v);
            T *y = static_cast<T *>(Y);
            if (x_format == PV_MX_E2M1) return launch_direct<kE2M1, kE2M1>(ctx, w, x, nblk, y);
            return launch_direct<kE2M1, kE4M3>(ctx, w, x, nblk, y);
        });
    }
    // scratch: scales with rows of whole words; the splits' sums
    const int64_t pitch = (nblk + 3) & ~3;
    const bool pad = pitch != nblk;
    // (f32 of E4M3: in_features below 2^23 as the interface has it, its rows half as long as that limit)
    pv_status st = check_pitch(ctx, x.pitch * (x_format == PV_MX_E4M3 && y_type == PV_F32 ? 2 : 1));
    if (st != PV_OK) return st;
    const size_t wb = round16(pad ? (size_t)(out * pitch) : 0), xb = round16(pad ? (size_t)(tokens * pitch) : 0);
    void *scratch = nullptr;
    if (wb + xb + c.partial) {
        st = pv_ops_scratch(ctx, wb + xb + c.partial, &scratch);
        if (st != PV_OK) return st;
    }
    uint8_t *ws = static_cast<uint8_t *>(scratch), *xs = ws + wb;
    float *partial = reinterpret_cast<float *>(xs + xb);
    pv_timed t(ctx, PV_K_MX_PRODUCT);
    if (pad) {
        auto words = [&](const uint8_t *from, int64_t rows, uint8_t *to) {
            const int64_t blocks = (rows * (pitch / 4) + 255) / 256;
            if (!pv_grid_fits(blocks, 256)) return pv_fail(ctx, PV_ERR_UNSUPPORTED, "too many scales");
            hipLaunchKernelGGL(k_pad_scales, dim3((unsigned)blocks), dim3(256), 0, ctx->stream, from, rows, nblk, to, (int)pitch);
            PV_HIP(ctx, hipGetLastError());
            return PV_OK;
        };
        st = words(w_scales, out, ws);
        if (st == PV_OK) st = words(x_scales, tokens, xs);
        if (st != PV_OK) return st;
        w.scales = ws;
        x.scales = xs;
    }
    return pv_for_dtype(y_type, [&](auto v) {
        using T = decltype(v);
        T *y = static_cast<T *>(Y);
        if (x_format == PV_MX_E2M1) return launch<kE2M1, kE2M1>(ctx, c, w, x, nblk, pitch, partial, y);
        return launch<kE2M1, kE4M3>(ctx, c, w, x, nblk, pitch, partial, y);
    });
}

pv_status pv_launch_mx_product_grads(pv_ctx *ctx, int64_t tokens, int64_t out, int64_t in, int x_format,
                                     const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *w_codes,
                                     const uint8_t *w_scales, const void *dY, int dx_type, void *dX, float *dW)
{
    const int64_t tp = padded(tokens), op = padded(out);
    const bool pad = dX && op != out;          // rows of dY that need an end
    pv_status st = check_pitch(ctx, 2 * (dX && dW ? (op > tp ? op : tp) : dX ? op : tp));
    if (st != PV_OK) return st;
    const choice cx = choose<kBF16, kBF16>(in, tokens, (int)(op / 32)), cw = choose<kBF16, kBF16>(in, out, (int)(tp / 32));
    // in order: the sums of either gradient | W^T, dY with padded rows | X^T, dY^T
    const size_t sums = round16(dX && cx.partial > (dW ? cw.partial : 0) ? cx.partial : dW ? cw.partial : 0);
    const int64_t wt = dX ? in * op : 0, dyp = pad ? tokens * op : 0, xt = dW ? in * tp : 0, dyt = dW ? out * tp : 0;
    void *p;
    st = pv_ops_scratch(ctx, sums + (size_t)(wt + dyp + xt + dyt) * 2, &p);
    if (st != PV_OK) return st;
    float *partial = static_cast<float *>(p);
    pv_bf16 *WT = reinterpret_cast<pv_bf16 *>(static_cast<uint8_t *>(p) + sums), *DYP = WT + wt, *XT = DYP + dyp, *DYT = XT + xt;
    pv_timed t(ctx, PV_K_MX_PRODUCT);
    turned m[3];
    int n = 0;
    if (dX) m[n++] = turn(kE2M1, w_codes, w_scales, out, in, WT);
    if (dW) m[n++] = turn(x_format, x_codes, x_scales, tokens, in, XT);
    if (dW) m[n++] = turn(kBF16, dY, nullptr, tokens, out, DYT);
    if ((st = transpose(ctx, m, n)) != PV_OK) return st;
    if (dX) {
        if (pad) {
            const int64_t blocks = (tokens * (op / 8) + 255) / 256;
            if (!pv_grid_fits(blocks, 256)) return pv_fail(ctx, PV_ERR_UNSUPPORTED, "too many rows of dY");
            hipLaunchKernelGGL(k_pad_rows, dim3((unsigned)blocks), dim3(256), 0, ctx->stream, static_cast<const pv_bf16 *>(dY),
                               tokens, out, DYP, op);
            PV_HIP(ctx, hipGetLastError());
        }
        const operand w = plain(WT, in, op), x = plain(pad ? DYP : dY, tokens, op);
        st = pv_for_dtype(dx_type, [&](auto v) {
            using T = decltype(v);
            return launch<kBF16, kBF16>(ctx, cx, w, x, (int)(op / 32), 0, partial, static_cast<T *>(dX));
        });
        if (st != PV_OK) return st;
    }
    if (dW) {
        st = launch<kBF16, kBF16>(ctx, cw, plain(XT, in, tp), plain(DYT, out, tp), (int)(tp / 32), 0, partial, dW);
    }
    return st;
}
