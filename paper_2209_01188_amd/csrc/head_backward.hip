// Backward of the LM head: da = G E (G fp32 [M, V] the gradient of the logits, E fp16 [V, H] the embedding matrix where the
// client keeps it), then the derivative of the final LayerNorm.  Three launches: G to fp16 tiles, the product in blocks with the
// contraction split, the sums of the splits with the LayerNorm.
//
// 2048 x 250880 x 4096: 540 + 3340 to 3700 + 30 us (1140 to 1260 TFLOP/s in the product, by the clock that the card's power leaves;
// an fp16 library product of this size alone 3360); 351 x 50257 x 2560: 22 + 105 + 12; 24 x 250880 x 14336: 14 + 1260 + 16, 5.7 TB/s
// of E; 16 x 50257 x 1024: 6 + 18 + 7.
#include <mutex>

#include "../../include/petals_finetune.h"
#include "../../include/petals_span.h"
#include "client_internal.h"
#include "common.h"
#include "host_util.h"
#include "ln_backward.h"
#include "span_internal.h"

namespace {

typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));     // rows of an odd vocabulary begin anywhere

// G as fp16 in the operand order of v_mfma_f32_16x16x32_f16: tile (mt, kt) of 16 rows x 32 columns is 1 KB, lane slot
// 16 (column / 8) + row holds 8 columns.  A row's section is scaled so that its largest value becomes 32768: fp16 then rounds
// by at most 2^-11 of a value down to 2^-29 of the largest (a softmax's gradient reaches from 1 down to 1e-9 and less), and the largest,
// mostly the label's, exactly.  lo (may be null): what the rounding left, in the same scale.
// A wave per row and section, SKT k-tiles: it reads 1 KB of the row at a time (a row of an odd vocabulary begins anywhere; the
// tiles' own 128 bytes of it would touch two lines each), takes the maximum, and drops its halves into LDS where the tiles lie;
// from there they go out as whole tiles of 16 rows.  Bound by its bytes: 5.7 TB/s at 2048 x 250880.  272 bytes from one group of 8 columns to the next, so that the 64 lanes'
// halves fall on different banks.
constexpr int PACK_GROUP = 16 * 16 + 16, PACK_TILE = 4 * PACK_GROUP;
constexpr int head_section_kt(bool pair) { return pair ? 32 : 64; }
template <bool PAIR>
__global__ void __launch_bounds__(1024) k_head_pack(const float *__restrict__ G, int M, int V, int KT, int sections,
                                                    __half *__restrict__ hi, __half *__restrict__ lo, float *__restrict__ unit) {
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int SKT = head_section_kt(PAIR), STEPS = SKT / 8;
    const int mt = __builtin_amdgcn_readfirstlane(blockIdx.x / sections), sec = blockIdx.x - mt * sections, MTT = (M + 15) >> 4;
    const int lane = threadIdx.x & 63, r = threadIdx.x >> 6, t = mt * 16 + r, v0 = sec * SKT * 32 + lane * 4;
    const float *row = G + (size_t)min(t, M - 1) * V;
    float f[STEPS][4];
    float mx = 0.0f;
#pragma unroll
    for (int i = 0; i < STEPS; i++) {
        const int v = v0 + i * 256;
        if (v + 3 < V) {
            const v4f a = __builtin_nontemporal_load((const v4f_any *)(row + v));
#pragma unroll
            for (int e = 0; e < 4; e++) f[i][e] = a[e];
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++) f[i][e] = v + e < V ? row[v + e] : 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < STEPS; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) mx = fmaxf(mx, fabsf(f[i][e]));
    mx = wave_max(mx);
    // (rows behind the call's, sections of zeros and of next to nothing: a unit of 2^-60, so that the ratio of two units stays a number)
    const float u = t < M ? fmaxf(mx * 0x1p-15f, 0x1p-60f) : 0x1p-60f, s = t < M ? 1.0f / u : 0.0f;
    if (lane == 0) unit[(size_t)sec * MTT * 16 + t] = u;
    unsigned char *mine = lds + (lane >> 3) * PACK_TILE + ((lane & 7) >> 1) * PACK_GROUP + r * 16 + (lane & 1) * 8;
#pragma unroll
    for (int i = 0; i < STEPS; i++) {
        v4h h, l;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float x = f[i][e] * s;
            h[e] = (_Float16)x;
            l[e] = (_Float16)(x - (float)h[e]);
        }
        *(v4h *)(mine + i * 8 * PACK_TILE) = h;
        if (PAIR) *(v4h *)(mine + (SKT + i * 8) * PACK_TILE) = l;
    }
    __syncthreads();
    const int at = (lane >> 4) * PACK_GROUP + (lane & 15) * 16;
#pragma unroll
    for (int i = r; i < SKT; i += 16) {
        const int kt = sec * SKT + i;
        if (kt >= KT) break;
        const size_t to = (((size_t)mt * KT + kt) * 64 + lane) * 8;
        *(v8h *)(hi + to) = *(const v8h *)(lds + i * PACK_TILE + at);
        if (PAIR) *(v8h *)(lo + to) = *(const v8h *)(lds + (SKT + i) * PACK_TILE + at);
    }
}

// The product: output blocks of BM tokens x 256 columns, 8 waves of BM / 2 x 64, the contraction over the vocabulary split over
// workgroups until every compute unit has one.  Token tiles and 32 rows x 512 bytes of E are copied to a ring of slots in LDS,
// NSLOT - 1 stages ahead (rings of 5 and 6 slots, which fit as well: no gain).  Eight waves, because a wave has 256 registers in two to
// a SIMD: four of 128 x 128 would read a third less of LDS, but did not keep their sums in registers.  The contraction runs along E's columns in memory, so its operands are turned around: a lane reads 4 columns
// of 8 rows and makes of them, one byte permutation per word, the A operands of 4 products (product i has columns 4 a + i).
// PAIR: the token tiles twice, G's values and what their rounding left; calls of up to 64 rows, which wait for E's bytes anyway.
// Full blocks are bound by the matrix instructions (69 % of the cycles busy, at the 1.7 GHz that their power leaves) and close to it
// by LDS (256 x 256: 1024 cycles of each to a stage); with one round of blocks (351 x 50257 x 2560, 192 x 256) a stage takes 790 ns.
constexpr int NSLOT = 4;
template <int BM, bool PAIR>
__global__ void __launch_bounds__(512, 2) k_head_block(const __half *__restrict__ E, const __half *__restrict__ hi, const __half *__restrict__ lo,
                                                       const float *__restrict__ unit, int M, int V, int H, int KT, int nb_m,
                                                       int nb_n, int kt_per, float *__restrict__ part) {
    constexpr int BN = 256, TM = BM / 32, TN = 4;               // tiles of 16 per wave: tokens, columns
    constexpr int GT = BM / 16, GS = PAIR ? 8 : GT, SLOT = 16384 + GS * 1024, GL = (GS + 7) / 8, LOADS = 2 + GL;
    constexpr int FULL = GS % 8 ? GS % 8 : 8;                   // waves that copy GL token tiles per stage, the others one less
    constexpr int section_kt = head_section_kt(PAIR);
    static_assert(!PAIR || 2 * GT <= 8, "a token tile for every wave");
    extern __shared__ __align__(16) unsigned char lds[];
    // workgroup -> block: an XCD (every eighth workgroup) takes a run of blocks of one split, four along the tokens at a time.
    // (Divisions are done by the vector unit; what is worked out from them is to be scalar all the same.)
    const int blocks = gridDim.x, xcd = blockIdx.x & 7, per = blocks >> 3, rest = blocks & 7;
    const int ord = xcd * per + min(xcd, rest) + (blockIdx.x >> 3), split = __builtin_amdgcn_readfirstlane(ord / (nb_m * nb_n)), in = ord - split * nb_m * nb_n;
    const int strip = __builtin_amdgcn_readfirstlane(in / (4 * nb_n)), wide = min(4, nb_m - 4 * strip), of_strip = in - strip * 4 * nb_n;
    const int bn = __builtin_amdgcn_readfirstlane(of_strip / wide), bm = strip * 4 + of_strip - bn * wide;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
    const int k0 = split * kt_per, k1 = min(KT, k0 + kt_per), MTT = (M + 15) >> 4;

    // what this wave copies per stage: rows 4 wave .. + 4 of E, two per instruction, and GL token tiles (fewer than 8 tiles of a
    // pair: some waves copy one that nobody reads).  The buffer form: rows behind the matrix come as zeros.  The 128-byte halves
    // of a row's 256 change places in every other octet of rows, so that the octets that are read together lie in different banks.
    const uint32_t e_off = ((uint32_t)((wave * 4 + (lane >> 5)) * H) + (uint32_t)min(bn * BN + ((lane & 31) ^ (8 * ((wave >> 1) & 1))) * 8, H - 8)) * 2;
    const auto copy = [&](const void *base, uint32_t bytes, uint32_t off, int at) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)bytes, 0x00020000),
                                                 (__attribute__((address_space(3))) void *)(lds + at), 16, (int)off, 0, 0, 0);
    };
    const auto copies = [&](int kt, int slot) {
        const int k = min(kt, k1 - 1), v = min(k * 32, V), rows = __builtin_amdgcn_readfirstlane(min(32, V - v));     // (k-tiles that fill up the last four have none)
#pragma unroll
        for (int i = 0; i < 2; i++) copy(E + (size_t)v * H, (uint32_t)rows * H * 2, e_off + i * 4u * H, slot * SLOT + (wave * 4 + 2 * i) * 512);
#pragma unroll
        for (int i = 0; i < GL; i++) {
            const int tile = wave + 8 * i;
            if (FULL < 8 && i == GL - 1 && wave >= FULL) break;
            copy((PAIR && tile >= GT ? lo : hi) + ((size_t)min(bm * GT + (PAIR ? tile % GT : tile), MTT - 1) * KT + k) * 512, 1024, lane * 16,
                 slot * SLOT + 16384 + tile * 1024);
        }
    };
    // operands: row 8 (lane / 16) + i, columns 64 wn + 4 (lane % 16) .. + 4; token tile j
    const int e_at = (lane >> 4) * 8 * 512 + ((wn * 128 + (lane & 15) * 8) ^ (128 * ((lane >> 4) & 1))), g_at = 16384 + wm * TM * 1024 + lane * 16;
    const auto read_e = [&](int slot, int i) { return *(const v2i *)(lds + slot * SLOT + e_at + i * 512); };
    const auto read_g = [&](int slot, int j) { return *(const v8h *)(lds + slot * SLOT + g_at + (j < TM ? j : GT + j - TM) * 1024); };

    v4f acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
        for (int j = 0; j < TM; j++) acc[i][j] = v4f{0, 0, 0, 0};
    // the units of a section's rows, two sections at a time in LDS behind the ring
    const int rows = MTT * 16;
    const auto copy_units = [&](int kt) {
        const int sec = kt / section_kt;
        if (wave == 0) copy(unit + (size_t)sec * rows, rows * 4, bm * BM * 4 + lane * 16, NSLOT * SLOT + (sec & 1) * 1024);
    };
    const auto unit_of = [&](int j, int kt) { return *(const float *)(lds + NSLOT * SLOT + ((kt / section_kt) & 1) * 1024 + ((wm * TM + j) * 16 + (lane & 15)) * 4); };
    copy_units(k0);
    copy_units(min(k0 + section_kt, KT - 1));
#pragma unroll
    for (int s = 0; s < NSLOT; s++) copies(k0 + s, s);
    v2i fe[2][8];
    constexpr int NG = PAIR ? 2 * TM : TM;
    v8h fg[2][NG];
    // at most `behind` stages' copies of this wave still on their way, its LDS reads done
    const auto wait = [&](auto BEHIND) {
        constexpr int behind = decltype(BEHIND)::value;
        if (FULL < 8 && wave >= FULL) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(behind * (LOADS - 1)) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(behind * LOADS) : "memory");
    };
    wait(std::integral_constant<int, NSLOT - 1>());
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; i++) fe[0][i] = read_e(0, i);
#pragma unroll
    for (int j = 0; j < NG; j++) fg[0][j] = read_g(0, j);
    wait(std::integral_constant<int, NSLOT - 2>());
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");

    // Stage kt: its operands are in registers, everybody has read its slot, and everybody's copies for stage kt + 1 have
    // landed.  Beside the products, the copies of stage kt + NSLOT are requested and the operands of kt + 1 read, a few at a time.
    const auto stage = [&](int kt, auto S) {
        constexpr int free_slot = decltype(S)::value, next_slot = (free_slot + 1) % NSLOT, cur = free_slot & 1, nxt = cur ^ 1;
        const auto beside = [&](int at) {                        // after eighth `at` of the products
            __builtin_amdgcn_sched_barrier(0);
            if (at == 0) copies(kt + NSLOT, free_slot);
            if (at == 1 || at == 2) {
#pragma unroll
                for (int r = 0; r < 4; r++) fe[nxt][4 * (at - 1) + r] = read_e(next_slot, 4 * (at - 1) + r);
            }
            if (at == 3 || at == 4) {
#pragma unroll
                for (int r = at == 3 ? 0 : (NG + 1) / 2; r < (at == 3 ? (NG + 1) / 2 : NG); r++) fg[nxt][r] = read_g(next_slot, r);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
#pragma unroll
        for (int i = 0; i < TN; i++) {
            v4i a;
#pragma unroll
            for (int w = 0; w < 4; w++)
                a[w] = (int)__builtin_amdgcn_perm((uint32_t)fe[cur][2 * w + 1][i >> 1], (uint32_t)fe[cur][2 * w][i >> 1], i & 1 ? 0x07060302 : 0x05040100);
            const v8h av = *(const v8h *)&a;
#pragma unroll
            for (int j = 0; j < TM; j++) {
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av, fg[cur][j], acc[i][j], 0, 0, 0);
                if constexpr (PAIR) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av, fg[cur][TM + j], acc[i][j], 0, 0, 0);
                if (TM == 1 || j == TM / 2 - 1) beside(2 * i);
                if (j == TM - 1) beside(2 * i + 1);
            }
        }
        wait(std::integral_constant<int, NSLOT - 2>());
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    for (int kt = k0; kt < k1; kt += 4) {
        if (!(kt & (section_kt - 1)) && kt > k0) {                   // the next section has its own unit
#pragma unroll
            for (int j = 0; j < TM; j++) {
                const float ratio = unit_of(j, kt - section_kt) / unit_of(j, kt);
#pragma unroll
                for (int i = 0; i < TN; i++) acc[i][j] *= ratio;
            }
            lds_barrier();                                       // everybody has read the section before: the one behind takes its place
            copy_units(min(kt + section_kt, KT - 1));
        }
        stage(kt, std::integral_constant<int, 0>());
        stage(kt + 1, std::integral_constant<int, 1>());
        stage(kt + 2, std::integral_constant<int, 2>());
        stage(kt + 3, std::integral_constant<int, 3>());
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // nothing may land in LDS after the workgroup's end
    // result register r of tile (i, j): token lane % 16, column 4 (4 (lane / 16) + r) + i of the wave's
#pragma unroll
    for (int j = 0; j < TM; j++) {
        const int t = (bm * GT + wm * TM + j) * 16 + (lane & 15);
        if (t >= M) continue;
        const float u = unit[(size_t)((k1 - 1) / section_kt) * rows + t];
        float *o = part + ((size_t)split * M + t) * H;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const int c = bn * BN + wn * 64 + (lane >> 4) * 16 + r * 4;
            if (c < H) *(v4f *)(o + c) = v4f{acc[0][j][r], acc[1][j][r], acc[2][j][r], acc[3][j][r]} * u;
        }
    }
}

// the partial sums of a row in order, then the LayerNorm
template <int NT, int PER>
__global__ void __launch_bounds__(NT) k_head_finish(const float *__restrict__ part, int splits, int M, int H, const __half *__restrict__ x,
                                                    const __half *__restrict__ g, float eps, __half *__restrict__ out) {
    __shared__ double sm[NT / 64][4];
    const int t = blockIdx.x;
    LnRow<PER> lr;
    ln_load<NT, PER>(lr, x + (size_t)t * H, g, H);
    float acc[PER][8] = {};
    add_rows<NT, PER, float, 8 / PER>(acc, splits, threadIdx.x * 8, H, [&](int s) { return part + ((size_t)s * M + t) * H; });
    ln_backward<NT, PER>(acc, lr, H, eps, sm);
    ln_store<NT, PER>(acc, out + (size_t)t * H, H);
}

// How a call of M rows is cut up, and where things lie in its store
struct HeadPlan {
    int mtt, kt, sections;           // token tiles, k-tiles (a multiple of 4), sections of a row
    bool pair;
    int bm, nb_m, nb_n;              // tokens of a block, blocks
    int kt_per, splits;
    size_t hi, lo, unit, part, bytes;
};
HeadPlan head_plan(const petals_client_config &cfg, int M) {
    constexpr int UNITS = 256;       // compute units: one workgroup each
    HeadPlan p;
    p.mtt = (M + 15) / 16;
    p.kt = (cfg.vocab + 127) / 128 * 4;
    p.pair = M <= PETALS_HEAD_BACKWARD_PAIR_ROWS;
    p.sections = (p.kt + head_section_kt(p.pair) - 1) / head_section_kt(p.pair);
    p.nb_n = (cfg.hidden + 255) / 256;
    // Tokens of a block and splits of the contraction: the fewest stages one after the other, each at what it takes (ns; measured at 351
    // rows x 50257 x 2560 and 768 x 100003 x 4096), and the partial sums' way to memory and back, 8 bytes of each at 2.4 TB/s.  (With 520
    // for 128 tokens and 9.6 TB/s, without 160: 300 rows x 50257 x 4096 190 us instead of 175, 1024 x 60000 x 14336 1763 instead of 1650,
    // 512 x 50257 x 1024 113 instead of 101.  Blocks of 224 tokens spill: 400 x 50257 x 4096 193 instead of 181.)
    const int shapes[4][2] = {{128, 560}, {160, 650}, {192, 750}, {256, 860}}, one[1][2] = {{M <= 32 ? 32 : 64, 500}};
    const int(*shape)[2] = p.pair ? one : shapes;
    double best = 0.0;
    for (int i = 0; i < (p.pair ? 1 : 4); i++) {
        const int nb_m = (M + shape[i][0] - 1) / shape[i][0], blocks = nb_m * p.nb_n;
        int before = 0;
        for (int rounds = 1; rounds <= 8; rounds++) {
            const int want = min((long long)UNITS * rounds / blocks, (long long)p.kt / 4);
            if (want <= before) continue;
            before = want;
            const int kt_per = (p.kt / 4 + want - 1) / want * 4, splits = (p.kt + kt_per - 1) / kt_per;
            const double ns = (double)(((long long)blocks * splits + UNITS - 1) / UNITS) * kt_per * shape[i][1] + splits * (double)M * cfg.hidden / 300.0;
            if (best == 0.0 || ns < best) {
                best = ns;
                p.bm = shape[i][0];
                p.nb_m = nb_m;
                p.kt_per = kt_per;
                p.splits = splits;
            }
            if (p.pair) break;
        }
        if (!before) {                // more blocks than eight rounds hold
            const double ns = (double)((blocks + UNITS - 1) / UNITS) * p.kt * shape[i][1] + (double)M * cfg.hidden / 300.0;
            if (best == 0.0 || ns < best) {
                best = ns;
                p.bm = shape[i][0];
                p.nb_m = nb_m;
                p.kt_per = p.kt;
                p.splits = 1;
            }
        }
    }
    const size_t tiles = ps_align_up((size_t)p.mtt * p.kt * 1024);
    p.hi = 0;
    p.lo = tiles;
    p.unit = p.lo + (p.pair ? tiles : 0);
    p.part = p.unit + ps_align_up((size_t)p.mtt * 16 * p.sections * sizeof(float));
    p.bytes = p.part + ps_align_up((size_t)p.splits * M * cfg.hidden * sizeof(float));
    return p;
}

// The limit of a kernel's dynamic LDS belongs to the function on a GPU, for the whole process: set once for each
struct LdsLimit {
    static constexpr int MOST = 64;
    std::mutex lock;
    bool set[MOST] = {};
    hipError_t allow(const void *kernel, int bytes) {
        int gpu = 0;
        if (hipError_t e = hipGetDevice(&gpu)) return e;
        std::lock_guard<std::mutex> hold(lock);
        if (gpu < MOST && set[gpu]) return hipSuccess;
        const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (gpu < MOST) set[gpu] = e == hipSuccess;
        return e;
    }
};

template <bool PAIR>
hipError_t head_pack(const HeadPlan &p, const float *G, uint8_t *store, int M, int V, hipStream_t st) {
    constexpr int bytes = head_section_kt(PAIR) * PACK_TILE * (PAIR ? 2 : 1);
    static LdsLimit limit;
    if (hipError_t e = limit.allow((const void *)k_head_pack<PAIR>, bytes)) return e;
    k_head_pack<PAIR><<<p.sections * p.mtt, 1024, bytes, st>>>(G, M, V, p.kt, p.sections, (__half *)(store + p.hi), (__half *)(store + p.lo),
                                                               (float *)(store + p.unit));
    return hipGetLastError();
}
template <int BM, bool PAIR>
hipError_t head_block(const HeadPlan &p, const __half *E, uint8_t *store, int M, int V, int H, hipStream_t st) {
    constexpr int bytes = NSLOT * (16384 + (PAIR ? 8 : BM / 16) * 1024) + 2048;
    static LdsLimit limit;
    if (hipError_t e = limit.allow((const void *)k_head_block<BM, PAIR>, bytes)) return e;
    k_head_block<BM, PAIR><<<p.nb_m * p.nb_n * p.splits, 512, bytes, st>>>(E, (const __half *)(store + p.hi), (const __half *)(store + p.lo),
                                                                          (const float *)(store + p.unit), M, V, H, p.kt, p.nb_m,
                                                                          p.nb_n, p.kt_per, (float *)(store + p.part));
    return hipGetLastError();
}

int check_rows(const petals_client_config &cfg, int32_t M) {
    if (M < 1) return ps_fail(PETALS_ERR_INVALID_ARG, "M must be positive");
    if (M > cfg.max_rows_per_call) return ps_fail(PETALS_ERR_CAPACITY, "%d rows exceed max_rows_per_call %d", M, cfg.max_rows_per_call);
    if (M > PETALS_BACKWARD_ROWS_MAX) return ps_fail(PETALS_ERR_UNSUPPORTED, "%d rows exceed %d", M, PETALS_BACKWARD_ROWS_MAX);
    if (cfg.vocab > 1 << 30) return ps_fail(PETALS_ERR_UNSUPPORTED, "vocabulary %d exceeds 2^30", cfg.vocab);
    return PETALS_OK;
}

}  // namespace

extern "C" {

int petals_client_lm_head_backward_bytes(const petals_client_config *cfg, int32_t M, size_t *bytes) {
    if (!bytes) return ps_fail(PETALS_ERR_INVALID_ARG, "null pointer");
    if (int rc = ps_check_client_config(cfg)) return rc;
    if (int rc = check_rows(*cfg, M)) return rc;
    *bytes = head_plan(*cfg, M).bytes;
    return PETALS_OK;
}

int petals_client_lm_head_backward(petals_client *client, void *dev_store, const void *hidden_in, const float *grad_logits, int32_t M,
                                   void *grad_hidden_out, void *stream) {
    if (!client || !dev_store || !hidden_in || !grad_logits || !grad_hidden_out) return ps_fail(PETALS_ERR_INVALID_ARG, "null pointer");
    if ((uintptr_t)dev_store & 255) return ps_fail(PETALS_ERR_INVALID_ARG, "store must be 256-byte aligned");
    const ps_client_view c = ps_view(client);
    if (int rc = check_rows(*c.cfg, M)) return rc;
    if (grad_hidden_out == hidden_in || grad_hidden_out == (const void *)grad_logits)
        return ps_fail(PETALS_ERR_INVALID_ARG, "buffers alias");
    const HeadPlan p = head_plan(*c.cfg, M);
    const int V = c.cfg->vocab, H = c.cfg->hidden;
    uint8_t *store = (uint8_t *)dev_store;
    hipStream_t st = (hipStream_t)stream;
    const __half *E = (const __half *)c.p->embeddings, *x = (const __half *)hidden_in, *g = (const __half *)c.p->final_ln_g;
    __half *out = (__half *)grad_hidden_out;
    const float *part = (const float *)(store + p.part);
    hipError_t e = p.pair ? head_pack<true>(p, grad_logits, store, M, V, st) : head_pack<false>(p, grad_logits, store, M, V, st);
    HIP_TRY(e);
    e = p.bm == 32    ? head_block<32, true>(p, E, store, M, V, H, st)
        : p.bm == 64  ? head_block<64, true>(p, E, store, M, V, H, st)
        : p.bm == 128 ? head_block<128, false>(p, E, store, M, V, H, st)
        : p.bm == 160 ? head_block<160, false>(p, E, store, M, V, H, st)
        : p.bm == 192 ? head_block<192, false>(p, E, store, M, V, H, st)
                      : head_block<256, false>(p, E, store, M, V, H, st);
    HIP_TRY(e);
    if (H <= 2048) k_head_finish<256, 1><<<M, 256, 0, st>>>(part, p.splits, M, H, x, g, c.cfg->ln_eps, out);
    else if (H <= 4096) k_head_finish<512, 1><<<M, 512, 0, st>>>(part, p.splits, M, H, x, g, c.cfg->ln_eps, out);
    else if (H <= 8192) k_head_finish<1024, 1><<<M, 1024, 0, st>>>(part, p.splits, M, H, x, g, c.cfg->ln_eps, out);
    else k_head_finish<1024, 2><<<M, 1024, 0, st>>>(part, p.splits, M, H, x, g, c.cfg->ln_eps, out);
    HIP_TRY(hipGetLastError());
    return PETALS_OK;
}

}  // extern "C"
