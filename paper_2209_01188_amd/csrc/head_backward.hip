// Backward of the LM head: da = G E (G fp32 [M, V] the gradient of the logits, E fp16 [V, H] the embedding matrix where the
// client keeps it), then the derivative of the final LayerNorm.
#include "../../include/petals_finetune.h"
#include "../../include/petals_span.h"
#include "client_internal.h"
#include "common.h"
#include "host_util.h"
#include "ln_backward.h"
#include "span_internal.h"

namespace {

constexpr int SECTION = 4096;              // columns of G that share a row's scale
constexpr int SECTION_KT = SECTION / 32;   // in k-tiles
constexpr int CHUNK = 128;                 // columns of E that a wave owns
typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));     // rows of an odd vocabulary begin anywhere

// G as fp16 in the operand order of v_mfma_f32_16x16x32_f16: tile (mt, kt) of 16 rows x 32 columns is 1 KB, lane slot
// 16 (column / 8) + row holds 8 columns.  A row's section is scaled so that its largest value becomes 32768: fp16 then keeps
// 2^-12 of a value down to 2^-29 of the largest (a softmax's gradient reaches from 1 down to 1e-9 and less), and the largest,
// mostly the label's, exactly.  lo (may be null): what the rounding left, in the same scale.
// One workgroup per 16 rows and section, a wave per row.
__global__ void __launch_bounds__(1024) k_head_pack(const float *__restrict__ G, int M, int V, int KT, int sections,
                                                    __half *__restrict__ hi, __half *__restrict__ lo, float *__restrict__ unit) {
    const int sec = blockIdx.x, mt = blockIdx.y, lane = threadIdx.x & 63, r = threadIdx.x >> 6, t = mt * 16 + r;
    float f[SECTION / 512][8];
    float mx = 0.0f;
#pragma unroll
    for (int i = 0; i < SECTION / 512; i++) {
        const int v = sec * SECTION + i * 512 + lane * 8;
        const float *row = G + (size_t)min(t, M - 1) * V;
        if (v + 7 < V) {
            const v4f a = *(const v4f_any *)(row + v), b = *(const v4f_any *)(row + v + 4);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                f[i][e] = a[e];
                f[i][4 + e] = b[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) f[i][e] = v + e < V ? row[v + e] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 8; e++) mx = fmaxf(mx, fabsf(f[i][e]));
    }
    mx = t < M ? wave_max(mx) : 0.0f;
    // (sections of zeros and of next to nothing: a unit of 2^-60, so that the ratio of two units stays a number)
    const float u = fmaxf(mx * 0x1p-15f, 0x1p-60f), s = 1.0f / u;
    if (lane == 0) unit[(size_t)t * sections + sec] = u;
#pragma unroll
    for (int i = 0; i < SECTION / 512; i++) {
        const int kt = sec * SECTION_KT + i * 16 + (lane >> 2);
        if (kt >= KT) continue;
        v8h h, l;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float x = t < M ? f[i][e] * s : 0.0f;
            h[e] = (_Float16)x;
            l[e] = (_Float16)(x - (float)h[e]);
        }
        const size_t at = (((size_t)mt * KT + kt) * 64 + (lane & 3) * 16 + r) * 8;
        *(v8h *)(hi + at) = h;
        if (lo) *(v8h *)(lo + at) = l;
    }
}

// A wave owns 128 columns of E and walks the rows 32 at a time: a lane loads 8 rows x 8 columns (16 bytes per row; 16 lanes
// cover 256 consecutive bytes) and turns them around in registers, one byte permutation per word, into the A operands of 8
// products: product j has columns 8 a + j, a = 0..15.  The token tiles are the B operand.
template <int MT, bool PAIR>
__global__ void __launch_bounds__(512) k_head_rows(const __half *__restrict__ E, const __half *__restrict__ hi, const __half *__restrict__ lo,
                                                   const float *__restrict__ unit, int M, int V, int H, int KT, int sections, int kt_per,
                                                   float *__restrict__ part) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int col = (blockIdx.x * waves + wave) * CHUNK + (lane & 15) * 8, mt0 = blockIdx.z * MT;
    const int k0 = blockIdx.y * kt_per, k1 = min(KT, k0 + kt_per);
    const __half *Ec = E + min(col, H - 8);
    const int MTT = (M + 15) >> 4;
    v4f acc[MT][8];
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
        for (int j = 0; j < 8; j++) acc[m][j] = v4f{0, 0, 0, 0};
    float u[MT];
#pragma unroll
    for (int m = 0; m < MT; m++) u[m] = unit[(size_t)(min(mt0 + m, MTT - 1) * 16 + (lane & 15)) * sections + k0 / SECTION_KT];
    for (int kt = k0; kt < k1; kt++) {
        if (kt % SECTION_KT == 0 && kt > k0) {                   // the next section has its own unit
#pragma unroll
            for (int m = 0; m < MT; m++) {
                const float next = unit[(size_t)(min(mt0 + m, MTT - 1) * 16 + (lane & 15)) * sections + kt / SECTION_KT], q = u[m] / next;
#pragma unroll
                for (int j = 0; j < 8; j++) acc[m][j] *= q;
                u[m] = next;
            }
        }
        v4i r[8];
#pragma unroll
        for (int i = 0; i < 8; i++) r[i] = *(const v4i *)(Ec + (size_t)min(kt * 32 + (lane >> 4) * 8 + i, V - 1) * H);
        v8h b[MT], bl[MT];
#pragma unroll
        for (int m = 0; m < MT; m++) {
            const size_t at = (((size_t)min(mt0 + m, MTT - 1) * KT + kt) * 64 + lane) * 8;
            b[m] = *(const v8h *)(hi + at);
            if (PAIR) bl[m] = *(const v8h *)(lo + at);
        }
#pragma unroll
        for (int j = 0; j < 8; j++) {
            v4i a;
#pragma unroll
            for (int w = 0; w < 4; w++)
                a[w] = (int)__builtin_amdgcn_perm((uint32_t)r[2 * w + 1][j >> 1], (uint32_t)r[2 * w][j >> 1], j & 1 ? 0x07060302 : 0x05040100);
            const v8h av = *(const v8h *)&a;
#pragma unroll
            for (int m = 0; m < MT; m++) {
                acc[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av, b[m], acc[m][j], 0, 0, 0);
                if (PAIR) acc[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av, bl[m], acc[m][j], 0, 0, 0);
            }
        }
    }
    // result register r of product j: token lane % 16, column 8 (4 (lane / 16) + r) + j of the wave's
    const int c0 = (blockIdx.x * waves + wave) * CHUNK + (lane >> 4) * 32;
#pragma unroll
    for (int m = 0; m < MT; m++) {
        const int t = (mt0 + m) * 16 + (lane & 15);
        if (t >= M) continue;
        float *o = part + ((size_t)blockIdx.y * M + t) * H + c0;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            if (c0 + 8 * r >= H) continue;
            *(v4f *)(o + 8 * r) = v4f{acc[m][0][r], acc[m][1][r], acc[m][2][r], acc[m][3][r]} * u[m];
            *(v4f *)(o + 8 * r + 4) = v4f{acc[m][4][r], acc[m][5][r], acc[m][6][r], acc[m][7][r]} * u[m];
        }
    }
}

// the partial sums of a row in order, then the LayerNorm
template <int NT, int PER>
__global__ void __launch_bounds__(NT) k_head_finish(const float *__restrict__ part, int splits, int M, int H, const __half *__restrict__ x,
                                                    const __half *__restrict__ g, float eps, __half *__restrict__ out) {
    __shared__ double sm[NT / 64][2];
    const int t = blockIdx.x;
    LnRow<PER> lr;
    ln_load<NT, PER>(lr, x + (size_t)t * H, g, H);
    float acc[PER][8] = {};
    for (int s = 0; s < splits; s++) {
        const float *row = part + ((size_t)s * M + t) * H;
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const int k = (threadIdx.x + i * NT) * 8;
            if (k < H) {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const v4f f = *(const v4f *)(row + k + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[i][4 * h + e] += f[e];
                }
            }
        }
    }
    ln_backward<NT, PER>(acc, lr, H, eps, sm);
    ln_store<NT, PER>(acc, out + (size_t)t * H, H);
}

// How a call of M rows is cut up, and where things lie in its store
struct HeadPlan {
    int mtt, kt, sections;           // token tiles, k-tiles, sections of a row
    bool pair;
    int mt, waves, groups, kt_per, splits;
    size_t hi, lo, unit, part, bytes;
};
HeadPlan head_plan(const petals_client_config &cfg, int M) {
    HeadPlan p;
    p.mtt = (M + 15) / 16;
    p.kt = (cfg.vocab + 31) / 32;
    p.sections = (cfg.vocab + SECTION - 1) / SECTION;
    p.pair = M <= PETALS_HEAD_BACKWARD_PAIR_ROWS;
    p.mt = p.mtt >= 4 ? 4 : p.mtt == 3 ? 4 : p.mtt;
    const int chunks = (cfg.hidden + CHUNK - 1) / CHUNK;
    p.groups = (chunks + 7) / 8;
    p.waves = (chunks + p.groups - 1) / p.groups;
    const int want = max(1, 512 / (p.groups * ((p.mtt + p.mt - 1) / p.mt)));
    p.kt_per = max(4, (p.kt + want - 1) / want);
    p.splits = (p.kt + p.kt_per - 1) / p.kt_per;
    const size_t tiles = ps_align_up((size_t)p.mtt * p.kt * 1024);
    p.hi = 0;
    p.lo = tiles;
    p.unit = p.lo + (p.pair ? tiles : 0);
    p.part = p.unit + ps_align_up((size_t)p.mtt * 16 * p.sections * sizeof(float));
    p.bytes = p.part + ps_align_up((size_t)p.splits * M * cfg.hidden * sizeof(float));
    return p;
}

template <int MT>
void head_rows(const HeadPlan &p, const __half *E, uint8_t *store, int M, int V, int H, hipStream_t st) {
    const dim3 grid(p.groups, p.splits, (p.mtt + MT - 1) / MT);
    const __half *hi = (const __half *)(store + p.hi), *lo = (const __half *)(store + p.lo);
    const float *unit = (const float *)(store + p.unit);
    float *part = (float *)(store + p.part);
    if (p.pair) k_head_rows<MT, true><<<grid, 64 * p.waves, 0, st>>>(E, hi, lo, unit, M, V, H, p.kt, p.sections, p.kt_per, part);
    else k_head_rows<MT, false><<<grid, 64 * p.waves, 0, st>>>(E, hi, lo, unit, M, V, H, p.kt, p.sections, p.kt_per, part);
}

}  // namespace

extern "C" {

int petals_client_lm_head_backward_bytes(const petals_client_config *cfg, int32_t M, size_t *bytes) {
    if (!bytes) return ps_fail(PETALS_ERR_INVALID_ARG, "null pointer");
    if (int rc = ps_check_client_config(cfg)) return rc;
    if (M < 1) return ps_fail(PETALS_ERR_INVALID_ARG, "M must be positive");
    if (M > cfg->max_rows_per_call) return ps_fail(PETALS_ERR_CAPACITY, "%d rows exceed max_rows_per_call %d", M, cfg->max_rows_per_call);
    *bytes = head_plan(*cfg, M).bytes;
    return PETALS_OK;
}

int petals_client_lm_head_backward(petals_client *client, void *dev_store, const void *hidden_in, const float *grad_logits, int32_t M,
                                   void *grad_hidden_out, void *stream) {
    if (!client || !dev_store || !hidden_in || !grad_logits || !grad_hidden_out) return ps_fail(PETALS_ERR_INVALID_ARG, "null pointer");
    if ((uintptr_t)dev_store & 255) return ps_fail(PETALS_ERR_INVALID_ARG, "store must be 256-byte aligned");
    const ps_client_view c = ps_view(client);
    if (M < 1) return ps_fail(PETALS_ERR_INVALID_ARG, "M must be positive");
    if (M > c.cfg->max_rows_per_call) return ps_fail(PETALS_ERR_CAPACITY, "%d rows exceed max_rows_per_call %d", M, c.cfg->max_rows_per_call);
    if (grad_hidden_out == hidden_in || grad_hidden_out == (const void *)grad_logits)
        return ps_fail(PETALS_ERR_INVALID_ARG, "buffers alias");
    const HeadPlan p = head_plan(*c.cfg, M);
    const int V = c.cfg->vocab, H = c.cfg->hidden;
    uint8_t *store = (uint8_t *)dev_store;
    hipStream_t st = (hipStream_t)stream;
    const __half *E = (const __half *)c.p->embeddings, *x = (const __half *)hidden_in, *g = (const __half *)c.p->final_ln_g;
    __half *out = (__half *)grad_hidden_out;
    const float *part = (const float *)(store + p.part);
    k_head_pack<<<dim3(p.sections, p.mtt), 1024, 0, st>>>(grad_logits, M, V, p.kt, p.sections, (__half *)(store + p.hi),
                                                          p.pair ? (__half *)(store + p.lo) : nullptr, (float *)(store + p.unit));
    HIP_TRY(hipGetLastError());
    if (p.mt == 1) head_rows<1>(p, E, store, M, V, H, st);
    else if (p.mt == 2) head_rows<2>(p, E, store, M, V, H, st);
    else head_rows<4>(p, E, store, M, V, H, st);
    HIP_TRY(hipGetLastError());
    if (H <= 2048) k_head_finish<256, 1><<<M, 256, 0, st>>>(part, p.splits, M, H, x, g, c.cfg->ln_eps, out);
    else if (H <= 4096) k_head_finish<512, 1><<<M, 512, 0, st>>>(part, p.splits, M, H, x, g, c.cfg->ln_eps, out);
    else if (H <= 8192) k_head_finish<1024, 1><<<M, 1024, 0, st>>>(part, p.splits, M, H, x, g, c.cfg->ln_eps, out);
    else k_head_finish<1024, 2><<<M, 1024, 0, st>>>(part, p.splits, M, H, x, g, c.cfg->ln_eps, out);
    HIP_TRY(hipGetLastError());
    return PETALS_OK;
}

}  // extern "C"
