// C ABI of libspd: model object over caller-owned buffers and the orchestration of
// one decoder forward (verify step / draft step / prefill) out of the HIP kernels.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <mutex>
#include <new>
#include <string>
#include <vector>

#include "../../include/spd.h"
#include "launch.h"

using namespace spd;

namespace {

thread_local char g_err[512] = "";

int32_t fail(int32_t code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
int32_t fail(int32_t code, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return code;
}

#define HIP_TRY(expr)                                                                          \
    do {                                                                                       \
        hipError_t e_ = (expr);                                                                \
        if (e_ != hipSuccess)                                                                  \
            return fail(SPD_ERR_HIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e_),    \
                        __FILE__, __LINE__);                                                   \
    } while (0)

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }


struct Layout {                    // byte offsets inside the three buffers
    // packed
    size_t embed, lm_head, final_norm;
    std::vector<size_t> attn_norm, wqkv, wo, mlp_norm, wgu, wdown;
    size_t packed_total;
    // kv
    size_t kv_layer_stride, kv_k_bytes, kv_v_bytes, kv_total;
    int v_stride;
    // workspace
    size_t h, qkv, xn, xo, xf, rope, logits, ssq_a, ssq_b, d_lens, d_error, qa_count, qa_abort, part, arrive, zero, chain;
    size_t ph, pqkv, pxn, pxo, pxf, pssq_a, pssq_b, ppart;      // prefill passes of up to prefill_rows rows
    size_t pw, pwscale;             // matrices in 4 bits: one of them as the prompt kernels read it
    int prefill_rows, pssq_ld;      // pssq: [part][pssq_ld] of the rows
    size_t ws_total;
};

int32_t check_shape(const spd_model_config &c) {
    if (c.n_layers < 1 || c.d_model < 32 || c.n_heads < 1 || c.d_ffn < 8 || c.vocab < 16 ||
        c.max_seqs < 1 || c.max_positions < 1)
        return fail(SPD_ERR_SHAPE, "non-positive dimension in spd_model_config");
    if (c.d_model % 32) return fail(SPD_ERR_SHAPE, "d_model %d must be a multiple of 32", c.d_model);
    if (c.head_dim != 64 && c.head_dim != 128)
        return fail(SPD_ERR_SHAPE, "head_dim %d must be 64 or 128", c.head_dim);
    if ((c.n_heads * c.head_dim) % 32)
        return fail(SPD_ERR_SHAPE, "n_heads*head_dim must be a multiple of 32");
    if (c.d_ffn % 8) return fail(SPD_ERR_SHAPE, "d_ffn %d must be a multiple of 8", c.d_ffn);
    if (c.vocab % 16) return fail(SPD_ERR_SHAPE, "vocab %d must be a multiple of 16", c.vocab);
    if (c.max_seqs > SPD_MAX_ROWS) return fail(SPD_ERR_SHAPE, "max_seqs %d exceeds %d", c.max_seqs, SPD_MAX_ROWS);
    if (!(c.rms_eps >= 0.f) || !(c.rope_theta > 0.f)) return fail(SPD_ERR_SHAPE, "bad rms_eps / rope_theta");
    return SPD_OK;
}

// q4_group: 0 for matrices in bf16, else the group size of matrices in 4 bits
void make_layout(const spd_model_config &c, int q4_group, Layout &L) {
    auto matrix_bytes = [&](int N, int K) { return q4_group ? q4_packed_bytes(N, K, q4_group) : packed_matrix_bytes(N, K); };
    const int d = c.d_model, HD = c.n_heads * c.head_dim, F = c.d_ffn, V = c.vocab;
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, 256); return o; };
    L.embed = take((size_t)V * d * 2);
    L.lm_head = take(matrix_bytes(V, d));
    L.final_norm = take((size_t)d * 4);
    for (int l = 0; l < c.n_layers; ++l) {
        L.attn_norm.push_back(take((size_t)d * 4));
        L.wqkv.push_back(take(matrix_bytes(3 * HD, d)));
        L.wo.push_back(take(matrix_bytes(d, HD)));
        L.mlp_norm.push_back(take((size_t)d * 4));
        L.wgu.push_back(take(matrix_bytes(2 * F, d)));
        L.wdown.push_back(take(matrix_bytes(d, F)));
    }
    L.packed_total = off;

    L.v_stride = (c.max_positions + 31) / 32 * 32;         // V is stored transposed, rows padded to 32 positions
    L.kv_k_bytes = (size_t)c.max_seqs * c.n_heads * c.max_positions * c.head_dim * 2;
    L.kv_v_bytes = (size_t)c.max_seqs * c.n_heads * c.head_dim * L.v_stride * 2;
    L.kv_layer_stride = align_up(L.kv_k_bytes, 256) + align_up(L.kv_v_bytes, 256);
    L.kv_total = L.kv_layer_stride * c.n_layers;

    off = 0;
    const size_t KSd = d / 32, KShd = HD / 32, KSf = (F + 31) / 32;
    L.h = take((size_t)kMaxRows * d * 4);
    L.qkv = take((size_t)kMaxRows * 3 * HD * 4);
    L.xn = take((size_t)kMaxGroups * KSd * 1024);
    L.xo = take((size_t)kMaxGroups * KShd * 1024);
    L.xf = take((size_t)kMaxGroups * KSf * 1024);
    L.rope = take((size_t)c.max_positions * (c.head_dim / 2) * 2 * 4);
    L.logits = take((size_t)kMaxRows * V * 4);
    L.d_lens = take((size_t)kMaxRows * 4);
    L.d_error = take(4);
    L.qa_count = take((size_t)c.n_heads * 4);
    L.qa_abort = take(4);
    L.ssq_a = take((size_t)(d / 16) * kMaxRows * 4);
    L.ssq_b = take((size_t)(d / 16) * kMaxRows * 4);
    size_t pb = attention_partial_bytes(c.head_dim);         // (shared: attention and the projections run one after the other)
    for (size_t b : {gemm_batch_scratch_bytes(3 * HD, d), gemm_batch_scratch_bytes(d, HD), gemm_batch_scratch_bytes(2 * F, d),
                     gemm_batch_scratch_bytes(d, F), gemm_batch_scratch_bytes(V, d)})
        pb = b > pb ? b : pb;
    if (q4_group)
        for (size_t b : {q4_workspace_bytes(kMaxRows, 3 * HD, d), q4_workspace_bytes(kMaxRows, d, HD), q4_workspace_bytes(kMaxRows, 2 * F, d),
                         q4_workspace_bytes(kMaxRows, d, F), q4_workspace_bytes(kMaxRows, V, d)})
            pb = b > pb ? b : pb;
    L.part = take(pb);
    L.arrive = take((size_t)kBatchMaxTileGroups * 4);
    L.zero = take(1024);
    L.chain = chain_shape_ok(d, HD, F) ? take(chain_bytes(d, HD, F)) : 0;
    // prefill: activations of one pass, whole row tiles of 16 rows (a workgroup tile may reach beyond the last one: the kernel
    // clamps the row tiles that it reads and writes no row that is not there)
    L.prefill_rows = std::min((int)kPrefillRows, c.max_positions);
    const size_t pr = align_up((size_t)L.prefill_rows, 16);
    L.pssq_ld = (int)pr;
    const size_t pssq_parts = (d / 16 + 3) / 4;
    L.ph = take(pr * d * 4);
    L.pqkv = take(pr * 3 * HD * 4);
    L.pxn = take(pr * KSd * 64 * kTerms);
    L.pxo = take(pr * KShd * 64 * kTerms);
    L.pxf = take(pr * KSf * 64 * kTerms);
    L.pssq_a = take(pr * pssq_parts * 4);
    L.pssq_b = take(pr * pssq_parts * 4);
    L.ppart = take(std::max({prefill_partial_bytes(3 * HD, L.prefill_rows), prefill_partial_bytes(d, L.prefill_rows), prefill_partial_bytes(2 * F, L.prefill_rows)}));
    L.pw = L.pwscale = 0;
    if (q4_group) {
        const size_t most = std::max({packed_matrix_bytes(3 * HD, d), packed_matrix_bytes(d, HD), packed_matrix_bytes(2 * F, d), packed_matrix_bytes(d, F)});
        L.pw = take(most);
        L.pwscale = take(most / 16);                       // a float for 16 rows and a K-step, where the block takes 1 KiB
    }
    L.ws_total = off;
}

GemmTuning default_tuning(int N, int K) {
    // Measured on MI355X at 5 rows: for K = 4096 (128 K-steps) the activation slice held in
    // registers and one persistent workgroup per CU is fastest, 8 waves x 16 steps for the
    // smaller matrices and 16 x 8 for the larger ones; otherwise fewer tiles -> more waves splitting K.
    int tiles = N / 16, KS = (K + 31) / 32;
    GemmTuning t;
    t.grid_cap = 0;
    t.ring = 8;
    t.no_regb = 0;
    t.no_batch = 0;
    t.force_batch = 0;
    if (KS == 128) t.waves = tiles >= 1024 ? 16 : 8;    // gate|up, LM head: 16 waves x 8 steps measured 1-2 % faster
    else if (KS == 64) t.waves = 8;
    else if (KS == 32) t.waves = 4;
    else if (tiles >= 1024) t.waves = 4;
    else if (tiles >= 512) t.waves = 8;
    else t.waves = 16;
    // One row group over a short K: the launch is a chain of latencies, and fewer waves shorten its reduction across waves.
    // Draft step of the 12-layer shape (d = 768), 4 / 8 / 16 waves for QKV, O and gate|up: 1 sequence 256.1 / 258.6 / 270.1 us,
    // 3 sequences 294.5 / 295.4 / 306.1, 5 sequences 319.7 / 312.1 / 321.4; its down projection (K = 2048), 4 / 8 waves: 252.9 /
    // 256.1.  The same order at d = 256, 512, 640, 896 and 2048.  Two row groups (6..10 rows) go best as they are.
    t.waves_few[0] = t.waves_few[1] = t.waves;
    if (KS <= 64) {
        t.waves_few[0] = 4;
        t.waves_few[1] = (KS == 64 || t.waves == 4) ? 4 : 8;
    }
    return t;
}

}  // namespace

// Bytes of a layer's packed matrices, and up to where a model counts as small: a layer fits the L2s (8 x 4 MiB) next to everything else.
static size_t layer_weight_bytes(const spd_model_config &c) {
    const int d = c.d_model, HD = c.n_heads * c.head_dim, F = c.d_ffn;
    return packed_matrix_bytes(3 * HD, d) + packed_matrix_bytes(d, HD) + packed_matrix_bytes(2 * F, d) + packed_matrix_bytes(d, F);
}
constexpr size_t kSmallLayer = (size_t)26 << 20;

struct spd_model {
    spd_model_config cfg;
    Layout L;
    char *packed, *kv, *ws;
    std::vector<int32_t> lens;         // KV lengths (host).  With dev_lens: only an upper bound
    std::vector<int32_t> lens_least;   // with dev_lens: what the lengths have at least (chooses kernels, bounds nothing)
    bool dev_lens = false;             // the kernels read the lengths from device memory (ws + L.d_lens)
    bool fuse_qa = false;              // QKV projection + attention as one kernel where the shape allows it
    bool fuse_qa2 = false;             // ... also for 6..8 rows of one sequence
    int chain = 0, chain_ok = 0;       // rows up to which all layers are one launch: as it is, and what shape and device allow
    bool fuse_qa_ok = false, fuse_qa2_ok = false;   // what the shape and the device allow (checked at creation)
    int q4_group = 0;                  // > 0: the matrices are held in 4 bits, with scales per group of so many columns
    int attn_slices = 0;               // workgroups per head of the stand-alone attention kernel (0: chosen by batch size)
    unsigned spin_limit = 1u << 22;    // polls before a wait between workgroups gives up
    std::vector<float> rope_host;
    GemmTuning t_qkv, t_o, t_gu, t_down, t_lm;
    // optional tracing: HIP events around every launch group of a forward
    struct Span { int kind; hipEvent_t a, b; };
    bool prof_on = false;
    std::vector<Span> spans;
    std::vector<hipEvent_t> pool;
    hipEvent_t take_event() {
        if (!pool.empty()) { hipEvent_t e = pool.back(); pool.pop_back(); return e; }
        hipEvent_t e = nullptr;
        if (hipEventCreate(&e) != hipSuccess) return nullptr;
        return e;
    }
    ~spd_model() {
        for (auto &sp : spans) { (void)hipEventDestroy(sp.a); (void)hipEventDestroy(sp.b); }
        for (auto e : pool) (void)hipEventDestroy(e);
    }
};

namespace {
enum ProfKind { PK_QKV = 0, PK_O, PK_GATE_UP, PK_DOWN, PK_LM_HEAD, PK_ATTENTION, PK_EMBED, PK_COUNT };

// Runs one launch group; when tracing is on, brackets it with events on the same stream (the interval
// then includes the dispatch of the group's first kernel).
#define PROF_TRY(kind, expr)                                                                   \
    do {                                                                                       \
        spd_model::Span sp_{(kind), nullptr, nullptr};                                         \
        if (m->prof_on) {                                                                      \
            sp_.a = m->take_event(); sp_.b = m->take_event();                                  \
            if (!sp_.a || !sp_.b) return fail(SPD_ERR_HIP, "hipEventCreate failed");           \
            HIP_TRY(hipEventRecord(sp_.a, st));                                                \
        }                                                                                      \
        HIP_TRY(expr);                                                                         \
        if (m->prof_on) { HIP_TRY(hipEventRecord(sp_.b, st)); m->spans.push_back(sp_); }       \
    } while (0)

// Same for a group that is a single kernel whose launch wrapper can hand the two events to the launch
// itself: they then time the kernel's execution alone, which is what a profiler reports for it.
#define PROF_KERNEL(kind, expr)                                                                \
    do {                                                                                       \
        spd_model::Span sp_{(kind), nullptr, nullptr};                                         \
        LaunchTiming lt_{nullptr, nullptr, false};                                             \
        if (m->prof_on) {                                                                      \
            sp_.a = m->take_event(); sp_.b = m->take_event();                                  \
            if (!sp_.a || !sp_.b) return fail(SPD_ERR_HIP, "hipEventCreate failed");           \
            lt_.start = sp_.a; lt_.stop = sp_.b;                                               \
            launch_timing() = &lt_;                                                            \
        }                                                                                      \
        hipError_t pe_ = (expr);                                                               \
        launch_timing() = nullptr;                                                             \
        HIP_TRY(pe_);                                                                          \
        if (m->prof_on) {                                                                      \
            if (!lt_.used) return fail(SPD_ERR_HIP, "internal: the launch did not take its timing events"); \
            m->spans.push_back(sp_);                                                           \
        }                                                                                      \
    } while (0)

// A projection.  Over one row group of a bf16 matrix it is a single kernel; more rows may take several passes.
#define PROF_GEMM(kind, g, epi, tuning)                                                        \
    do {                                                                                       \
        if (m->q4_group) PROF_TRY(kind, project_q4(m, g, epi, st));                            \
        else if (rows <= kGroupRows) PROF_KERNEL(kind, launch_gemm(g, epi, tuning, st));       \
        else PROF_TRY(kind, launch_gemm(g, epi, tuning, st));                                  \
    } while (0)

// the projection that `g` describes, its matrix held in 4 bits
hipError_t project_q4(const spd_model *m, const GemmArgs &g, Epilogue epi, hipStream_t st) {
    Q4GemmArgs a{};
    a.W = g.W; a.N = g.N; a.K = g.K; a.group = m->q4_group; a.rows = g.rows;
    a.X = g.X; a.x_kind = g.x_rows ? Q4_X_F32 : Q4_X_PACKED; a.ldx = g.K;
    a.Y = g.Y; a.ldy = g.ldy;
    a.ssq_in = g.ssq_in; a.ssq_in_parts = g.ssq_in_parts; a.eps = g.eps;
    a.gain_next = g.gain_next; a.Xnext = (float *)g.Xnext; a.ssq_out = g.ssq_out;
    a.Xout = (float *)g.Xout; a.K_out = g.K_out;
    a.workspace = m->ws + m->L.part;
    return launch_q4_gemm(a, epi, st);
}
}  // namespace



extern "C" {

const char *spd_last_error(void) { return g_err; }

}  // extern "C"

namespace {

int32_t model_bytes(const spd_model_config *cfg, int q4_group, size_t *packed_bytes, size_t *kv_bytes, size_t *workspace_bytes) {
    if (!cfg) return fail(SPD_ERR_INVALID_ARG, "NULL config");
    int32_t rc = check_shape(*cfg);
    if (rc) return rc;
    Layout L;
    make_layout(*cfg, q4_group, L);
    if (packed_bytes) *packed_bytes = L.packed_total;
    if (kv_bytes) *kv_bytes = L.kv_total;
    if (workspace_bytes) *workspace_bytes = L.ws_total;
    return SPD_OK;
}

bool complete(const spd_q4_matrix *w) { return w && w->q && w->scales; }

// Exactly one of w (matrices in bf16) and w4 (in 4 bits) is given.
int32_t create_model(const spd_model_config *cfg, const spd_weights *w, const spd_weights_q4 *w4, void *packed,
                     size_t packed_bytes, void *kv_cache, size_t kv_bytes, void *workspace,
                     size_t workspace_bytes, void *stream, spd_model **out) {
    int32_t rc = check_shape(*cfg);
    if (rc) return rc;
    if (((uintptr_t)packed | (uintptr_t)kv_cache | (uintptr_t)workspace) & 255)
        return fail(SPD_ERR_INVALID_ARG, "buffers must be 256-byte aligned");
    if (w && (!w->embed || !w->final_norm || !w->attn_norm || !w->wq || !w->wk || !w->wv || !w->wo ||
              !w->mlp_norm || !w->w_gate || !w->w_up || !w->w_down || (!cfg->tied_embeddings && !w->lm_head)))
        return fail(SPD_ERR_INVALID_ARG, "NULL weight pointer");
    if (w4 && (!w4->embed || !w4->final_norm || !w4->attn_norm || !w4->wq || !w4->wk || !w4->wv || !w4->wo ||
               !w4->mlp_norm || !w4->w_gate || !w4->w_up || !w4->w_down || !complete(&w4->lm_head)))
        return fail(SPD_ERR_INVALID_ARG, "NULL weight pointer");
    if (w4 && !q4_group_ok(w4->group)) return fail(SPD_ERR_SHAPE, "group %d must be 32, 64 or 128", w4->group);
    spd_model *m = new (std::nothrow) spd_model;
    if (!m) return fail(SPD_ERR_INVALID_ARG, "out of host memory");
    m->cfg = *cfg;
    m->q4_group = w4 ? w4->group : 0;
    make_layout(*cfg, m->q4_group, m->L);
    const Layout &L = m->L;
    if (packed_bytes < L.packed_total || kv_bytes < L.kv_total || workspace_bytes < L.ws_total) {
        delete m;
        return fail(SPD_ERR_CAPACITY, "buffer smaller than spd_model_bytes reports");
    }
    m->packed = (char *)packed;
    m->kv = (char *)kv_cache;
    m->ws = (char *)workspace;
    m->lens.assign(cfg->max_seqs, 0);
    hipStream_t st = (hipStream_t)stream;
    const int d = cfg->d_model, HD = cfg->n_heads * cfg->head_dim, F = cfg->d_ffn, V = cfg->vocab;

#define CREATE_TRY(expr)                                                                      \
    do {                                                                                       \
        hipError_t e_ = (expr);                                                                \
        if (e_ != hipSuccess) {                                                                \
            delete m;                                                                          \
            return fail(SPD_ERR_HIP, "%s failed: %s", #expr, hipGetErrorString(e_));           \
        }                                                                                      \
    } while (0)

    CREATE_TRY(hipMemcpyAsync(m->packed + L.embed, w ? w->embed : w4->embed, (size_t)V * d * 2, hipMemcpyDeviceToDevice, st));
    auto pack4 = [&](int mode, const spd_q4_matrix &a, const spd_q4_matrix &b, const spd_q4_matrix &c, int N, int K, size_t off) {
        const void *const q[3] = {a.q, b.q, c.q}, *const s[3] = {a.scales, b.scales, c.scales};
        return launch_q4_pack(q, s, mode, N, K, m->q4_group, m->packed + off, st);
    };
    const spd_q4_matrix none{nullptr, nullptr};
    if (w4) CREATE_TRY(pack4(PACK_PLAIN, w4->lm_head, none, none, V, d, L.lm_head));
    else CREATE_TRY(launch_pack_weight(cfg->tied_embeddings ? w->embed : w->lm_head, nullptr, nullptr, PACK_PLAIN,
                                       V, d, m->packed + L.lm_head, st));
    CREATE_TRY(hipMemcpyAsync(m->packed + L.final_norm, w ? w->final_norm : w4->final_norm, (size_t)d * 4, hipMemcpyDeviceToDevice, st));
    for (int l = 0; w4 && l < cfg->n_layers; ++l) {
        if (!w4->attn_norm[l] || !w4->mlp_norm[l] || !complete(&w4->wq[l]) || !complete(&w4->wk[l]) || !complete(&w4->wv[l]) ||
            !complete(&w4->wo[l]) || !complete(&w4->w_gate[l]) || !complete(&w4->w_up[l]) || !complete(&w4->w_down[l])) {
            delete m;
            return fail(SPD_ERR_INVALID_ARG, "NULL weight pointer in layer %d", l);
        }
        CREATE_TRY(hipMemcpyAsync(m->packed + L.attn_norm[l], w4->attn_norm[l], (size_t)d * 4, hipMemcpyDeviceToDevice, st));
        CREATE_TRY(hipMemcpyAsync(m->packed + L.mlp_norm[l], w4->mlp_norm[l], (size_t)d * 4, hipMemcpyDeviceToDevice, st));
        CREATE_TRY(pack4(PACK_CONCAT3, w4->wq[l], w4->wk[l], w4->wv[l], 3 * HD, d, L.wqkv[l]));
        CREATE_TRY(pack4(PACK_PLAIN, w4->wo[l], none, none, d, HD, L.wo[l]));
        CREATE_TRY(pack4(PACK_GATE_UP, w4->w_gate[l], w4->w_up[l], none, 2 * F, d, L.wgu[l]));
        CREATE_TRY(pack4(PACK_PLAIN, w4->w_down[l], none, none, d, F, L.wdown[l]));
    }
    for (int l = 0; w && l < cfg->n_layers; ++l) {
        if (!w->attn_norm[l] || !w->wq[l] || !w->wk[l] || !w->wv[l] || !w->wo[l] || !w->mlp_norm[l] ||
            !w->w_gate[l] || !w->w_up[l] || !w->w_down[l]) {
            delete m;
            return fail(SPD_ERR_INVALID_ARG, "NULL weight pointer in layer %d", l);
        }
        CREATE_TRY(hipMemcpyAsync(m->packed + L.attn_norm[l], w->attn_norm[l], (size_t)d * 4, hipMemcpyDeviceToDevice, st));
        CREATE_TRY(launch_pack_weight(w->wq[l], w->wk[l], w->wv[l], PACK_CONCAT3, 3 * HD, d, m->packed + L.wqkv[l], st));
        CREATE_TRY(launch_pack_weight(w->wo[l], nullptr, nullptr, PACK_PLAIN, d, HD, m->packed + L.wo[l], st));
        CREATE_TRY(hipMemcpyAsync(m->packed + L.mlp_norm[l], w->mlp_norm[l], (size_t)d * 4, hipMemcpyDeviceToDevice, st));
        CREATE_TRY(launch_pack_weight(w->w_gate[l], w->w_up[l], nullptr, PACK_GATE_UP, 2 * F, d, m->packed + L.wgu[l], st));
        CREATE_TRY(launch_pack_weight(w->w_down[l], nullptr, nullptr, PACK_PLAIN, d, F, m->packed + L.wdown[l], st));
    }
    // workspace starts cleared: the padding columns of the packed activation buffers must be zero;
    // the KV cache too: the attention kernel reads (and masks) whole 32-position units, so every
    // slot must hold a finite value
    CREATE_TRY(launch_fill_zero(m->ws, L.ws_total, st));
    CREATE_TRY(launch_fill_zero(m->kv, L.kv_total, st));
    // RoPE table: angle(pos, i) = pos * theta^(-2i/head_dim), computed in double
    const int half = cfg->head_dim / 2;
    m->rope_host.resize((size_t)cfg->max_positions * half * 2);
    for (int p = 0; p < cfg->max_positions; ++p)
        for (int i = 0; i < half; ++i) {
            double ang = (double)p * std::pow((double)cfg->rope_theta, -2.0 * i / cfg->head_dim);
            m->rope_host[((size_t)p * half + i) * 2 + 0] = (float)std::cos(ang);
            m->rope_host[((size_t)p * half + i) * 2 + 1] = (float)std::sin(ang);
        }
    CREATE_TRY(hipMemcpyAsync(m->ws + L.rope, m->rope_host.data(), m->rope_host.size() * 4, hipMemcpyHostToDevice, st));
#undef CREATE_TRY

    m->t_qkv = default_tuning(3 * HD, d);
    m->t_o = default_tuning(d, HD);
    m->t_gu = default_tuning(2 * F, d);
    m->t_down = default_tuning(d, F);
    m->t_lm = default_tuning(V, d);
    // QKV projection + attention as one kernel where the shape and the device allow it
    // (these and the launch of all layers read weights in bf16)
    m->fuse_qa_ok = w && qkv_attention_supported(cfg->d_model, cfg->n_heads, cfg->head_dim, 1, 1, 1);
    m->fuse_qa2_ok = m->fuse_qa_ok && qkv_attention_supported(cfg->d_model, cfg->n_heads, cfg->head_dim, 8, 1, 8);
    m->fuse_qa = m->fuse_qa_ok;
    m->fuse_qa2 = m->fuse_qa2_ok;
    // (a layer has to fit the L2s: with more weights a launch per projection keeps the memory busier)
    m->chain = m->chain_ok = w && layer_weight_bytes(*cfg) <= kSmallLayer && chain_supported(d, HD, F, cfg->head_dim) ? chain_rows(d, HD, F) : 0;
    *out = m;
    return SPD_OK;
}

}  // namespace

extern "C" {

int32_t spd_model_bytes(const spd_model_config *cfg, size_t *packed_bytes, size_t *kv_bytes,
                        size_t *workspace_bytes) {
    return model_bytes(cfg, 0, packed_bytes, kv_bytes, workspace_bytes);
}

int32_t spd_model_bytes_q4(const spd_model_config *cfg, int32_t group, size_t *packed_bytes, size_t *kv_bytes,
                           size_t *workspace_bytes) {
    if (!q4_group_ok(group)) return fail(SPD_ERR_SHAPE, "group %d must be 32, 64 or 128", group);
    return model_bytes(cfg, group, packed_bytes, kv_bytes, workspace_bytes);
}

int32_t spd_model_create(const spd_model_config *cfg, const spd_weights *w, void *packed,
                         size_t packed_bytes, void *kv_cache, size_t kv_bytes, void *workspace,
                         size_t workspace_bytes, void *stream, spd_model **out) {
    if (!cfg || !w || !packed || !kv_cache || !workspace || !out)
        return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_model_create");
    return create_model(cfg, w, nullptr, packed, packed_bytes, kv_cache, kv_bytes, workspace, workspace_bytes, stream, out);
}

int32_t spd_model_create_q4(const spd_model_config *cfg, const spd_weights_q4 *w, void *packed,
                            size_t packed_bytes, void *kv_cache, size_t kv_bytes, void *workspace,
                            size_t workspace_bytes, void *stream, spd_model **out) {
    if (!cfg || !w || !packed || !kv_cache || !workspace || !out)
        return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_model_create_q4");
    return create_model(cfg, nullptr, w, packed, packed_bytes, kv_cache, kv_bytes, workspace, workspace_bytes, stream, out);
}

int32_t spd_model_set_tuning(spd_model *m, const spd_tuning *t) {
    if (!m || !t) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_model_set_tuning");
    if (t->batch_kernel < 0 || t->batch_kernel > 2) return fail(SPD_ERR_INVALID_ARG, "batch_kernel must be 0, 1 or 2");
    if (t->separate_qkv_attention != 0 && t->separate_qkv_attention != 1) return fail(SPD_ERR_INVALID_ARG, "separate_qkv_attention must be 0 or 1");
    if (t->attention_slices != 0 && t->attention_slices != 1 && t->attention_slices != 2 && t->attention_slices != 4 &&
        t->attention_slices != 8)
        return fail(SPD_ERR_INVALID_ARG, "attention_slices must be 0, 1, 2, 4 or 8");
    GemmTuning *gt[SPD_N_PROJECTIONS] = {&m->t_qkv, &m->t_o, &m->t_gu, &m->t_down, &m->t_lm};
    for (int i = 0; i < SPD_N_PROJECTIONS; ++i) {
        const int w = t->gemm_waves[i];
        if (w != 0 && w != 4 && w != 8 && w != 16) return fail(SPD_ERR_INVALID_ARG, "gemm_waves must be 0, 4, 8 or 16");
        if (t->gemm_grid_cap[i] < 0 || t->gemm_grid_cap[i] > 65535) return fail(SPD_ERR_INVALID_ARG, "gemm_grid_cap out of range");
        if (t->gemm_ring[i] != 0 && t->gemm_ring[i] != 8 && t->gemm_ring[i] != 16) return fail(SPD_ERR_INVALID_ARG, "gemm_ring must be 0, 8 or 16");
    }
    const spd_model_config &c = m->cfg;
    const int d = c.d_model, HD = c.n_heads * c.head_dim, F = c.d_ffn, V = c.vocab;
    const int Ns[SPD_N_PROJECTIONS] = {3 * HD, d, 2 * F, d, V}, Ks[SPD_N_PROJECTIONS] = {d, HD, d, F, d};
    for (int i = 0; i < SPD_N_PROJECTIONS; ++i) {
        *gt[i] = default_tuning(Ns[i], Ks[i]);
        if (t->gemm_waves[i]) gt[i]->waves = gt[i]->waves_few[0] = gt[i]->waves_few[1] = t->gemm_waves[i];
        gt[i]->grid_cap = t->gemm_grid_cap[i];
        if (t->gemm_ring[i]) gt[i]->ring = t->gemm_ring[i];
        gt[i]->no_regb = t->gemm_general_kernel[i] ? 1 : 0;
        gt[i]->no_batch = t->batch_kernel == 2 ? 1 : 0;
        gt[i]->force_batch = t->batch_kernel == 1 ? 1 : 0;
    }
    const spd_tuning plain{};
    spd_tuning chosen = *t;
    chosen.wait_spin_limit = 0;
    m->chain = memcmp(&chosen, &plain, sizeof(plain)) == 0 ? m->chain_ok : 0;     // any choice among the separate kernels means those
    m->fuse_qa = t->separate_qkv_attention ? false : m->fuse_qa_ok;
    m->fuse_qa2 = t->separate_qkv_attention ? false : m->fuse_qa2_ok;
    m->attn_slices = t->attention_slices;
    m->spin_limit = t->wait_spin_limit ? t->wait_spin_limit : (1u << 22);
    return SPD_OK;
}

int32_t spd_model_destroy(spd_model *m) {
    delete m;
    return SPD_OK;
}

int32_t spd_kv_set_len(spd_model *m, const int32_t *len, int32_t n_seqs) {
    if (!m || !len) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_kv_set_len");
    if (n_seqs < 0 || n_seqs > m->cfg.max_seqs) return fail(SPD_ERR_CAPACITY, "n_seqs %d exceeds max_seqs %d", n_seqs, m->cfg.max_seqs);
    for (int i = 0; i < n_seqs; ++i) {
        if (len[i] < 0) return fail(SPD_ERR_INVALID_ARG, "negative KV length");
        if (len[i] > m->cfg.max_positions) return fail(SPD_ERR_CAPACITY, "KV length %d exceeds max_positions %d", len[i], m->cfg.max_positions);
    }
    if (m->dev_lens) return fail(SPD_ERR_INVALID_ARG, "KV lengths live on the device: call spd_kv_lens_from_device first");
    for (int i = 0; i < n_seqs; ++i) m->lens[i] = len[i];
    return SPD_OK;
}

int32_t spd_kv_lens_to_device(spd_model *m, void *stream) {
    if (!m) return fail(SPD_ERR_INVALID_ARG, "NULL model");
    HIP_TRY(hipMemcpyAsync(m->ws + m->L.d_lens, m->lens.data(), (size_t)m->cfg.max_seqs * 4, hipMemcpyHostToDevice, (hipStream_t)stream));
    HIP_TRY(launch_fill_zero(m->ws + m->L.d_error, 16, (hipStream_t)stream));
    HIP_TRY(hipStreamSynchronize((hipStream_t)stream));          // the host array may change right after this call
    m->dev_lens = true;
    m->lens_least = m->lens;
    return SPD_OK;
}

int32_t spd_kv_lens_from_device(spd_model *m, void *stream) {
    if (!m) return fail(SPD_ERR_INVALID_ARG, "NULL model");
    if (!m->dev_lens) return SPD_OK;
    std::vector<int32_t> tmp((size_t)m->cfg.max_seqs + 1);
    HIP_TRY(hipMemcpyAsync(tmp.data(), m->ws + m->L.d_lens, (size_t)m->cfg.max_seqs * 4, hipMemcpyDeviceToHost, (hipStream_t)stream));
    HIP_TRY(hipMemcpyAsync(&tmp[m->cfg.max_seqs], m->ws + m->L.d_error, 4, hipMemcpyDeviceToHost, (hipStream_t)stream));
    HIP_TRY(hipStreamSynchronize((hipStream_t)stream));
    m->dev_lens = false;
    const bool overflow = tmp[m->cfg.max_seqs] != 0;
    for (int i = 0; i < m->cfg.max_seqs; ++i) m->lens[i] = std::max(0, std::min(tmp[i], m->cfg.max_positions));
    if (overflow) return fail(SPD_ERR_CAPACITY, "a forward ran with a device KV length that left no room for its rows");
    return SPD_OK;
}

int32_t spd_device_status(spd_model *m, void *stream) {
    if (!m) return fail(SPD_ERR_INVALID_ARG, "NULL model");
    int32_t flags[2] = {0, 0};
    HIP_TRY(hipMemcpyAsync(&flags[0], m->ws + m->L.d_error, 4, hipMemcpyDeviceToHost, (hipStream_t)stream));
    HIP_TRY(hipMemcpyAsync(&flags[1], m->ws + m->L.qa_abort, 4, hipMemcpyDeviceToHost, (hipStream_t)stream));
    HIP_TRY(hipStreamSynchronize((hipStream_t)stream));
    if (flags[1]) return fail(SPD_ERR_HIP, "a wait between workgroups hit its spin limit: results since then are invalid");
    if (flags[0]) return fail(SPD_ERR_CAPACITY, "a forward ran with a device KV length that left no room for its rows");
    return SPD_OK;
}

int32_t spd_kv_export(spd_model *m, int32_t layer, int32_t seq, int32_t pos0, int32_t n, float *k_out, float *v_out, void *stream) {
    if (!m || !k_out || !v_out) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_kv_export");
    const spd_model_config &c = m->cfg;
    if (layer < 0 || layer >= c.n_layers || seq < 0 || seq >= c.max_seqs) return fail(SPD_ERR_INVALID_ARG, "layer / sequence index out of range");
    if (n < 1 || pos0 < 0 || pos0 + n > c.max_positions) return fail(SPD_ERR_CAPACITY, "positions %d..%d outside the cache (%d)", pos0, pos0 + n - 1, c.max_positions);
    const Layout &L = m->L;
    const char *kv_l = m->kv + (size_t)layer * L.kv_layer_stride;
    const char *k = kv_l + (size_t)seq * c.n_heads * c.max_positions * c.head_dim * 2;
    const char *v = kv_l + align_up(L.kv_k_bytes, 256) + (size_t)seq * c.n_heads * c.head_dim * L.v_stride * 2;
    HIP_TRY(launch_kv_export(k, v, c.n_heads, c.head_dim, c.max_positions, pos0, n, k_out, v_out, (hipStream_t)stream));
    return SPD_OK;
}

int32_t spd_kv_get_len(const spd_model *m, int32_t *len, int32_t n_seqs) {
    if (!m || !len) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_kv_get_len");
    if (n_seqs < 0 || n_seqs > m->cfg.max_seqs) return fail(SPD_ERR_CAPACITY, "n_seqs exceeds max_seqs");
    for (int i = 0; i < n_seqs; ++i) len[i] = m->lens[i];
    return SPD_OK;
}

}  // extern "C"

namespace {

// Final norm (folded in) and LM head on the packed rows that the last layer left
int32_t run_lm_head(spd_model *m, int rows, float *logits_out, hipStream_t st) {
    const spd_model_config &c = m->cfg;
    const Layout &L = m->L;
    GemmArgs g{};
    g.batch_partials = (float *)(m->ws + L.part); g.batch_arrive = (unsigned *)(m->ws + L.arrive); g.batch_zero = m->ws + L.zero;
    g.W = m->packed + L.lm_head; g.X = m->ws + L.xn; g.N = c.vocab; g.K = c.d_model; g.rows = rows; g.Y = logits_out; g.ldy = c.vocab;
    g.ssq_in = (float *)(m->ws + L.ssq_b); g.ssq_in_parts = c.d_model / 16; g.eps = c.rms_eps; g.x_rows = true;
    PROF_GEMM(PK_LM_HEAD, g, EPI_STORE, m->t_lm);
    return SPD_OK;
}

// All layers in one launch (small models, up to 5 rows); at: lengths as for run_layers
int32_t run_chain(spd_model *m, const AttnArgs &lens, int seq0, int n_seqs, int M, int longest, const int32_t *tokens, int token_stride, const float *embeds, hipStream_t st) {
    const spd_model_config &c = m->cfg;
    const Layout &L = m->L;
    ChainArgs a{};
    AttnArgs at = lens;
    at.rope = (const float *)(m->ws + L.rope);
    at.k_cache = m->kv + (size_t)seq0 * c.n_heads * c.max_positions * c.head_dim * 2;
    at.v_cache = m->kv + align_up(L.kv_k_bytes, 256) + (size_t)seq0 * c.n_heads * c.head_dim * L.v_stride * 2;
    at.n_seqs = n_seqs; at.M = at.Mq = M; at.m0 = 0; at.H = c.n_heads; at.dh = c.head_dim; at.max_positions = c.max_positions; at.v_stride = L.v_stride;
    a.wqkv = m->packed + L.wqkv[0]; a.wo = m->packed + L.wo[0]; a.wgu = m->packed + L.wgu[0]; a.wdown = m->packed + L.wdown[0];
    a.attn_norm = (const float *)(m->packed + L.attn_norm[0]); a.mlp_norm = (const float *)(m->packed + L.mlp_norm[0]); a.final_norm = (const float *)(m->packed + L.final_norm);
    a.layer_stride = c.n_layers > 1 ? L.wqkv[1] - L.wqkv[0] : 0;             // every layer takes the same sizes, each a multiple of 256
    a.kv_stride = L.kv_layer_stride;
    a.n_layers = c.n_layers; a.rows = n_seqs * M; a.d = c.d_model; a.HD = c.n_heads * c.head_dim; a.F = c.d_ffn;
    a.eps = c.rms_eps; a.inv_d = 1.0f / (float)c.d_model;
    a.words = m->ws + L.chain;
    a.x_final = (uint16_t *)(m->ws + L.xn); a.ssq_final = (float *)(m->ws + L.ssq_b);
    a.spin_limit = m->spin_limit; a.abort_flag = (int *)(m->ws + L.qa_abort);
    HIP_TRY(launch_chain(a, at, longest, m->packed + L.embed, tokens, token_stride, embeds, c.vocab, st));
    return SPD_OK;
}

// A forward over pages: the rows' keys and values go into them, and the rows' attention reads them.
struct PagedLayers {
    PagedAppendArgs append;              // of a layer but for its cache; queries are turned where they are
    PagedAttentionArgs attention;
    const spd_paged_cache *cache;        // [n_layers]
    float *rows;                         // float32 [rows][n_heads * head_dim]: the attention's results
};

// Layers first .. of the decoder for M new rows of each of sequences seq0 .. seq0 + n_seqs - 1, and the LM head (logits_out may be NULL).
// The input rows are in place: h, packed (h * attn_norm[first]) and their sums of squares (one part per row); `at` has the
// KV lengths; longest: the longest of them as far as the host can tell.  kv_cached (a prompt's last row): layer
// `first`'s key and value of the row are in the cache, and the length counts them; the sums are as exact as the prompt kernels'.
// pages (else NULL): see PagedLayers; `at` has nothing to say then.
int32_t run_layers(spd_model *m, int first, AttnArgs &at, int seq0, int n_seqs, int M, int longest, bool kv_cached, float *logits_out, hipStream_t st, PagedLayers *pages = nullptr) {
    const spd_model_config &c = m->cfg;
    const Layout &L = m->L;
    const int rows = n_seqs * M;
    const int d = c.d_model, HD = c.n_heads * c.head_dim, F = c.d_ffn;
    float *h = (float *)(m->ws + L.h);
    float *qkv = (float *)(m->ws + L.qkv);
    void *xn = m->ws + L.xn, *xo = m->ws + L.xo, *xf = m->ws + L.xf;

    float *ssq_a = (float *)(m->ws + L.ssq_a), *ssq_b = (float *)(m->ws + L.ssq_b);
    const int d_tiles = d / 16;
    auto gain_of = [&](size_t off) { return (const float *)(m->packed + off); };

    at.qkv = qkv;
    at.rope = (const float *)(m->ws + L.rope);
    at.xout = xo;
    at.n_seqs = n_seqs; at.M = M; at.H = c.n_heads; at.dh = c.head_dim; at.max_positions = c.max_positions;
    at.v_stride = L.v_stride;
    at.slices = m->attn_slices;
    at.partials = (float *)(m->ws + L.part); at.arrive = (unsigned *)(m->ws + L.arrive);

    // Small models, few rows: a projection lasts about as long as its first loads take, so the weights of the next ones are
    // brought into L2 meanwhile.
    const bool prefetch = !pages && !m->q4_group && rows <= 2 * kGroupRows && layer_weight_bytes(c) <= kSmallLayer;
    const bool fused = !pages && m->fuse_qa && n_seqs == 1 && (rows <= kGroupRows || (rows <= 8 && m->fuse_qa2));   // shapes checked at creation
    for (int l = first; l < c.n_layers; ++l) {
        // RMSNorm is folded into the projections: the producer of h (input rows / O / down
        // epilogue) leaves packed (h * gain) and per-tile sums of squares; the consumer
        // scales its accumulators by 1 / rms.
        char *kv_l = m->kv + (size_t)l * L.kv_layer_stride;
        at.k_cache = kv_l + (size_t)seq0 * c.n_heads * c.max_positions * c.head_dim * 2;
        at.v_cache = kv_l + align_up(L.kv_k_bytes, 256) + (size_t)seq0 * c.n_heads * c.head_dim * L.v_stride * 2;
        GemmArgs g{};
        g.batch_partials = (float *)(m->ws + L.part); g.batch_arrive = (unsigned *)(m->ws + L.arrive); g.batch_zero = m->ws + L.zero; g.fold = kv_cached;
        at.row_cached = kv_cached && l == first;
        if (fused && !at.row_cached) {
            QkvAttnArgs qa{};
            qa.W = m->packed + L.wqkv[l]; qa.X = xn; qa.K = d; qa.rows = rows;
            qa.ssq_in = ssq_b; qa.ssq_in_parts = l == first ? 1 : d_tiles; qa.eps = c.rms_eps;
            at.m0 = 0; at.Mq = M;
            qa.at = at;
            qa.head_count = (unsigned *)(m->ws + L.qa_count); qa.spin_limit = m->spin_limit;
            qa.abort_flag = (int *)(m->ws + L.qa_abort);
            PROF_KERNEL(PK_QKV, launch_qkv_attention(qa, st));
        } else {
            g.W = m->packed + L.wqkv[l]; g.X = xn; g.N = at.row_cached && !m->q4_group ? HD : 3 * HD; g.K = d; g.rows = rows; g.Y = qkv; g.ldy = 3 * HD;
            g.ssq_in = ssq_b; g.ssq_in_parts = l == first ? 1 : d_tiles; g.eps = c.rms_eps; g.x_rows = l != first;
            PROF_GEMM(PK_QKV, g, EPI_STORE, m->t_qkv);
            WeightPrefetch pf{};
            if (prefetch) {
                auto add = [&](size_t off, int N, int K) { pf.m[pf.n].w = m->packed + off; pf.m[pf.n].tiles = N / 16; pf.m[pf.n++].tile_bytes = (K + 31) / 32 * 1024; };
                add(L.wo[l], d, HD);
                add(L.wgu[l], 2 * F, d);
                add(L.wdown[l], d, F);
                if (l + 1 < c.n_layers) add(L.wqkv[l + 1], 3 * HD, d);
            }
            if (pages) {
                auto in_pages = [&]() -> hipError_t {
                    pages->append.c.k = pages->attention.c.k = pages->cache[l].k; pages->append.c.v = pages->attention.c.v = pages->cache[l].v;
                    pages->append.c.k_scale = pages->attention.c.k_scale = pages->cache[l].k_scale; pages->append.c.v_scale = pages->attention.c.v_scale = pages->cache[l].v_scale;
                    hipError_t rc = launch_paged_append(pages->append, st);
                    if (rc == hipSuccess) rc = launch_paged_attention(pages->attention, st);
                    if (rc == hipSuccess && !m->q4_group) rc = launch_pack_rows(pages->rows, rows, HD, xo, st);
                    return rc;
                };
                PROF_TRY(PK_ATTENTION, in_pages());
            }
            for (int m0 = 0; m0 < M && !pages; m0 += 8) {         // at most 8 queries per sequence and launch
                at.m0 = m0; at.Mq = std::min(8, M - m0);
                PROF_TRY(PK_ATTENTION, launch_attention(at, longest, m0 == 0 ? pf : WeightPrefetch{}, st));
            }
        }
        g = GemmArgs{};
        g.batch_partials = (float *)(m->ws + L.part); g.batch_arrive = (unsigned *)(m->ws + L.arrive); g.batch_zero = m->ws + L.zero; g.fold = kv_cached;
        g.W = m->packed + L.wo[l]; g.X = xo; g.N = d; g.K = HD; g.rows = rows; g.Y = h; g.ldy = d;
        if (pages && m->q4_group) { g.X = pages->rows; g.x_rows = true; }
        g.gain_next = gain_of(L.mlp_norm[l]); g.Xnext = xn; g.ssq_out = ssq_a;
        PROF_GEMM(PK_O, g, EPI_RESIDUAL, m->t_o);
        g = GemmArgs{};
        g.batch_partials = (float *)(m->ws + L.part); g.batch_arrive = (unsigned *)(m->ws + L.arrive); g.batch_zero = m->ws + L.zero; g.fold = kv_cached;
        g.W = m->packed + L.wgu[l]; g.X = xn; g.N = 2 * F; g.K = d; g.rows = rows; g.Xout = xf; g.K_out = F;
        g.ssq_in = ssq_a; g.ssq_in_parts = d_tiles; g.eps = c.rms_eps; g.x_rows = true;
        PROF_GEMM(PK_GATE_UP, g, EPI_SWIGLU, m->t_gu);
        g = GemmArgs{};
        g.batch_partials = (float *)(m->ws + L.part); g.batch_arrive = (unsigned *)(m->ws + L.arrive); g.batch_zero = m->ws + L.zero; g.fold = kv_cached;
        g.W = m->packed + L.wdown[l]; g.X = xf; g.N = d; g.K = F; g.rows = rows; g.Y = h; g.ldy = d;
        g.gain_next = gain_of(l + 1 < c.n_layers ? L.attn_norm[l + 1] : L.final_norm); g.Xnext = xn; g.ssq_out = ssq_b; g.x_rows = true;
        PROF_GEMM(PK_DOWN, g, EPI_RESIDUAL, m->t_down);
    }
    return logits_out ? run_lm_head(m, rows, logits_out, st) : SPD_OK;
}

// One decoder forward over M new rows for sequences seq0 .. seq0 + n_seqs - 1.
// Input rows come from token ids (embedding gather) or from embedding rows.
// max_m: SPD_MAX_M for the public calls; the prefill feeds one sequence up to 64 rows per pass.
int32_t forward(spd_model *m, const int32_t *tokens, int token_stride, const float *embeds, int seq0, int n_seqs, int M,
                float *logits_out, hipStream_t st, int max_m = SPD_MAX_M) {
    const spd_model_config &c = m->cfg;
    const Layout &L = m->L;
    const int rows = n_seqs * M;
    if (M < 1 || M > max_m) return fail(SPD_ERR_SHAPE, "M = %d must be in 1..%d", M, max_m);
    if (n_seqs < 1 || rows > SPD_MAX_ROWS) return fail(SPD_ERR_SHAPE, "n_seqs * M = %d must be in 1..%d", rows, SPD_MAX_ROWS);
    if (seq0 < 0 || seq0 + n_seqs > c.max_seqs) return fail(SPD_ERR_CAPACITY, "sequence index beyond max_seqs %d", c.max_seqs);
    if (M > c.max_positions) return fail(SPD_ERR_CAPACITY, "M = %d exceeds max_positions %d", M, c.max_positions);
    if (tokens && token_stride < M) return fail(SPD_ERR_INVALID_ARG, "token stride %d below M = %d", token_stride, M);
    AttnArgs at{};
    int longest = 0;                                     // positions cached, as far as the host can tell
    for (int s = 0; s < n_seqs; ++s) {
        int len = m->lens[seq0 + s];
        longest = std::max(longest, m->dev_lens ? m->lens_least[seq0 + s] : len);
        // lengths on the device: the host value is an upper bound and the kernels guard themselves
        if (!m->dev_lens && len + M > c.max_positions)
            return fail(SPD_ERR_CAPACITY, "KV cache overflow: sequence %d has %d positions, +%d > %d", seq0 + s, len, M, c.max_positions);
        at.lens.len[s] = len;
    }
    if (m->dev_lens) {
        at.d_lens = (const int32_t *)(m->ws + L.d_lens) + seq0;
        at.d_error = (int32_t *)(m->ws + L.d_error);
    }
    const int d = c.d_model;
    if (rows <= m->chain && chain_pays(d, c.n_heads * c.head_dim, c.d_ffn, c.head_dim, n_seqs, M, longest) && !m->prof_on) {      // (traced one by one: the launches of a layer)
        int32_t rc = run_chain(m, at, seq0, n_seqs, M, longest, tokens, tokens ? token_stride : M, embeds, st);
        if (rc == SPD_OK && logits_out) rc = run_lm_head(m, rows, logits_out, st);
        if (rc) return rc;
        if (m->dev_lens) HIP_TRY(launch_lens_add((int32_t *)(m->ws + L.d_lens) + seq0, n_seqs, M, st));
        for (int s = 0; s < n_seqs; ++s) m->lens[seq0 + s] = std::min(m->lens[seq0 + s] + M, c.max_positions);
        return SPD_OK;
    }
    // input rows -> h, packed (h * attn_norm[0]) and sum of squares (one part per row)
    PROF_TRY(PK_EMBED, launch_input_rows(m->packed + L.embed, tokens, M, tokens ? token_stride : M, embeds, rows, d, c.vocab,
                                         (const float *)(m->packed + L.attn_norm[0]), (float *)(m->ws + L.h), m->ws + L.xn, (float *)(m->ws + L.ssq_b), st));
    const int32_t rc = run_layers(m, 0, at, seq0, n_seqs, M, longest, false, logits_out, st);
    if (rc) return rc;
    if (m->dev_lens) HIP_TRY(launch_lens_add((int32_t *)(m->ws + L.d_lens) + seq0, n_seqs, M, st));
    for (int s = 0; s < n_seqs; ++s) m->lens[seq0 + s] = std::min(m->lens[seq0 + s] + M, c.max_positions);
    return SPD_OK;
}

// One prefill pass: M rows (at most L.prefill_rows) of sequence `seq` through all layers; last_logits (may be NULL)
// receives the logits of the last one.
//
// What leaves the last layer is the keys and values of all rows and the logits of one, so nothing else of it is computed
// for all rows: the projection makes K and V, and the last row goes through the layer and the LM head by the kernels of single rows
// with the K and V that the cache then has (they do not depend on whether logits were asked for).  Four 7B layers, 2047 rows
// 8.62 -> 6.99 ms, 640 rows 2.89 -> 2.42, 33 rows 0.708 -> 0.668; the 12-layer draft, 1472 rows 1.76 -> 1.67, the 4-layer draft 0.88 -> 0.73.
int32_t prefill_pass(spd_model *m, int32_t seq, const float *embeds, const int32_t *tokens, int M, float *last_logits, hipStream_t st) {
    const spd_model_config &c = m->cfg;
    const Layout &L = m->L;
    const int d = c.d_model, HD = c.n_heads * c.head_dim, F = c.d_ffn, V = c.vocab;
    float *h = (float *)(m->ws + L.ph), *qkv = (float *)(m->ws + L.pqkv);
    float *ssq_a = (float *)(m->ws + L.pssq_a), *ssq_b = (float *)(m->ws + L.pssq_b);
    void *xn = m->ws + L.pxn, *xo = m->ws + L.pxo, *xf = m->ws + L.pxf;
    auto gain_of = [&](size_t off) { return (const float *)(m->packed + off); };
    PROF_TRY(PK_EMBED, launch_prefill_rows(m->packed + L.embed, tokens, embeds, M, d, V, gain_of(L.attn_norm[0]), h, xn, ssq_b, L.pssq_ld, st));
    PrefillAttnArgs at{};
    at.qkv = qkv; at.rope = (const float *)(m->ws + L.rope); at.xout = xo;
    at.rows = M; at.H = c.n_heads; at.dh = c.head_dim; at.max_positions = c.max_positions; at.v_stride = L.v_stride;
    at.len = m->lens[seq];
    if (m->dev_lens) {
        at.d_len = (const int32_t *)(m->ws + L.d_lens) + seq;
        at.d_error = (int32_t *)(m->ws + L.d_error);
    }
    const int parts = prefill_ssq_parts(d / 16, M, m->q4_group != 0);
    // g.W: features first .. first + g.N - 1 of the packed matrix (N x g.K) at `off`
    auto weights = [&](PrefillGemmArgs &g, size_t off, int N, int first) -> hipError_t {
        if (!m->q4_group) { g.W = m->packed + off + packed_matrix_bytes(first, g.K); return hipSuccess; }
        g.W = m->ws + L.pw; g.wscale = (const float *)(m->ws + L.pwscale); g.group_steps = m->q4_group / kStepK;
        return launch_q4_unpack(m->packed + off, N, g.K, m->q4_group, first / kTileN, g.N / kTileN, m->ws + L.pw, (float *)(m->ws + L.pwscale), st);
    };
    auto project = [&](PrefillGemmArgs &g, size_t off, int N, int first, Epilogue epi) -> hipError_t {
        const hipError_t rc = weights(g, off, N, first);
        return rc != hipSuccess ? rc : launch_prefill_gemm(g, epi, st);
    };
    for (int l = 0; l < c.n_layers; ++l) {
        const bool last = l + 1 == c.n_layers;
        char *kv_l = m->kv + (size_t)l * L.kv_layer_stride;
        at.k_cache = kv_l + (size_t)seq * c.n_heads * c.max_positions * c.head_dim * 2;
        at.v_cache = kv_l + align_up(L.kv_k_bytes, 256) + (size_t)seq * c.n_heads * c.head_dim * L.v_stride * 2;
        const int q0 = last ? HD : 0;                     // the last layer's queries are not needed: features HD .. 3 HD - 1
        PrefillGemmArgs common{};
        common.rows = M; common.ssq_ld = L.pssq_ld; common.eps = c.rms_eps;
        common.partials = (float *)(m->ws + L.ppart); common.arrive = (unsigned *)(m->ws + L.arrive);
        PrefillGemmArgs g = common;
        g.X = xn; g.N = 3 * HD - q0; g.K = d; g.Y = qkv + q0; g.ldy = 3 * HD;
        g.ssq_in = ssq_b; g.ssq_parts = l == 0 ? prefill_row_parts(d) : parts;
        PROF_TRY(PK_QKV, project(g, L.wqkv[l], 3 * HD, q0, EPI_STORE));
        PROF_TRY(PK_ATTENTION, launch_prefill_attention(at, !last, st));
        if (last) break;
        g = common;
        g.X = xo; g.N = d; g.K = HD; g.Y = h; g.ldy = d;
        g.gain_next = gain_of(L.mlp_norm[l]); g.Xnext = xn; g.ssq_out = ssq_a;
        PROF_TRY(PK_O, project(g, L.wo[l], d, 0, EPI_RESIDUAL));
        g = common;
        g.X = xn; g.N = 2 * F; g.K = d; g.Xout = xf;
        g.ssq_in = ssq_a; g.ssq_parts = parts;
        PROF_TRY(PK_GATE_UP, project(g, L.wgu[l], 2 * F, 0, EPI_SWIGLU));
        g = common;
        g.X = xf; g.N = d; g.K = F; g.Y = h; g.ldy = d;
        g.gain_next = gain_of(L.attn_norm[l + 1]); g.Xnext = xn; g.ssq_out = ssq_b;
        PROF_TRY(PK_DOWN, project(g, L.wdown[l], d, 0, EPI_RESIDUAL));
    }
    int32_t *d_len = (int32_t *)(m->ws + L.d_lens) + seq;
    if (m->dev_lens) HIP_TRY(launch_lens_add(d_len, 1, M, st));
    if (last_logits) {
        const int l = c.n_layers - 1;
        HIP_TRY(launch_input_rows(nullptr, nullptr, 1, 1, h + (size_t)(M - 1) * d, 1, d, V, gain_of(L.attn_norm[l]), (float *)(m->ws + L.h), m->ws + L.xn,
                                  (float *)(m->ws + L.ssq_b), st));
        AttnArgs one{};
        one.lens.len[0] = m->lens[seq] + M;
        if (m->dev_lens) {
            one.d_lens = d_len;
            one.d_error = at.d_error;
        }
        const int32_t rc = run_layers(m, l, one, seq, 1, 1, one.lens.len[0], true, last_logits, st);
        if (rc) return rc;
    }
    m->lens[seq] = std::min(m->lens[seq] + M, c.max_positions);
    return SPD_OK;
}

int32_t prefill_common(spd_model *m, int32_t seq, const float *embeds, const int32_t *tokens, int32_t n_rows,
                       float *last_logits, hipStream_t st) {
    if (!m || (!embeds && !tokens)) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_prefill");
    if (n_rows < 1) return fail(SPD_ERR_INVALID_ARG, "n_rows must be positive");
    if (seq < 0 || seq >= m->cfg.max_seqs) return fail(SPD_ERR_CAPACITY, "sequence index %d beyond max_seqs %d", seq, m->cfg.max_seqs);
    if (m->lens[seq] + n_rows > m->cfg.max_positions)
        return fail(SPD_ERR_CAPACITY, "KV cache overflow in prefill: %d + %d > %d", m->lens[seq], n_rows, m->cfg.max_positions);
    float *scratch = (float *)(m->ws + m->L.logits);
    if (m->dev_lens) m->lens_least[seq] = std::min(m->lens_least[seq] + n_rows, m->cfg.max_positions);
    // passes through the prefill kernels, unless a kernel family was asked for (batch_kernel = 1 or 2)
    if (!m->t_qkv.no_batch && !m->t_qkv.force_batch) {
        const int min_rows = prefill_min_rows(m->cfg.d_model, m->q4_group != 0);
        while (n_rows >= min_rows) {
            const int M = std::min(n_rows, m->L.prefill_rows);
            const int32_t rc = prefill_pass(m, seq, embeds, tokens, M, M == n_rows ? last_logits : nullptr, st);
            if (rc) return rc;
            n_rows -= M;
            if (embeds) embeds += (size_t)M * m->cfg.d_model;
            else tokens += M;
        }
        if (n_rows == 0) return SPD_OK;
    }
    // what is left -- rows per pass over the weights: 64 through the batched projection kernel (measured 0.108 ms per row at the 7B
    // shape against 0.128 for passes of 40), 40 (8 row groups) through the K-splitting kernel otherwise
    const bool batched = m->L.part != 0 && !m->t_qkv.no_batch;
    const int pass_rows = batched ? SPD_MAX_ROWS : 8 * kGroupRows;
    for (int r0 = 0; r0 < n_rows; r0 += pass_rows) {
        int M = n_rows - r0 < pass_rows ? n_rows - r0 : pass_rows;
        bool last = r0 + M >= n_rows;
        int32_t rc = forward(m, tokens ? tokens + r0 : nullptr, M, embeds ? embeds + (size_t)r0 * m->cfg.d_model : nullptr,
                             seq, 1, M, (last && last_logits) ? scratch : nullptr, st, pass_rows);
        if (rc) return rc;
        if (last && last_logits)
            HIP_TRY(hipMemcpyAsync(last_logits, scratch + (size_t)(M - 1) * m->cfg.vocab, (size_t)m->cfg.vocab * 4,
                                   hipMemcpyDeviceToDevice, st));
    }
    return SPD_OK;
}

}  // namespace

extern "C" {

int32_t spd_trace_enable(spd_model *m, int32_t enable) {
    if (!m) return fail(SPD_ERR_INVALID_ARG, "NULL model");
    m->prof_on = enable != 0;
    return SPD_OK;
}

int32_t spd_trace_read(spd_model *m, int32_t n_kinds, double *ms_sum, int32_t *count) {
    if (!m || !ms_sum || !count || n_kinds < 1) return fail(SPD_ERR_INVALID_ARG, "bad argument to spd_trace_read");
    for (int i = 0; i < n_kinds; ++i) { ms_sum[i] = 0.0; count[i] = 0; }
    for (auto &sp : m->spans) {
        HIP_TRY(hipEventSynchronize(sp.b));
        float ms = 0.f;
        HIP_TRY(hipEventElapsedTime(&ms, sp.a, sp.b));
        if (sp.kind < n_kinds) { ms_sum[sp.kind] += ms; count[sp.kind] += 1; }
        m->pool.push_back(sp.a);
        m->pool.push_back(sp.b);
    }
    m->spans.clear();
    return SPD_OK;
}

int32_t spd_prefill(spd_model *m, int32_t seq, const float *embeds, int32_t n_rows, float *last_logits, void *stream) {
    if (!embeds) return fail(SPD_ERR_INVALID_ARG, "NULL embeds");
    return prefill_common(m, seq, embeds, nullptr, n_rows, last_logits, (hipStream_t)stream);
}

int32_t spd_prefill_tokens(spd_model *m, int32_t seq, const int32_t *tokens, int32_t n_rows, float *last_logits, void *stream) {
    if (!tokens) return fail(SPD_ERR_INVALID_ARG, "NULL tokens");
    return prefill_common(m, seq, nullptr, tokens, n_rows, last_logits, (hipStream_t)stream);
}

int32_t spd_verify_forward(spd_model *m, const int32_t *tokens, int32_t n_seqs, int32_t M, float *logits_out, void *stream) {
    if (!m || !tokens || !logits_out) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_verify_forward");
    return forward(m, tokens, M, nullptr, 0, n_seqs, M, logits_out, (hipStream_t)stream);
}

int32_t spd_draft_step_strided(spd_model *m, const int32_t *tokens_in, int32_t in_stride, int32_t n_seqs, int32_t n_in,
                               float temperature, const float *u_draft, int32_t u_stride, float *D_row_out,
                               size_t D_stride, int32_t *token_out, int32_t token_stride, void *stream) {
    if (!m || !tokens_in || !u_draft || !D_row_out || !token_out) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_draft_step");
    if (n_in < 1 || n_in > 2) return fail(SPD_ERR_SHAPE, "n_in = %d must be 1 or 2", n_in);
    if (!(temperature >= 0.f)) return fail(SPD_ERR_INVALID_ARG, "temperature must be >= 0");
    if (in_stride < n_in || u_stride < 1 || token_stride < 1 || D_stride < (size_t)m->cfg.vocab)
        return fail(SPD_ERR_INVALID_ARG, "strides must cover one sequence's entries");
    float *scratch = (float *)(m->ws + m->L.logits);
    int32_t rc = forward(m, tokens_in, in_stride, nullptr, 0, n_seqs, n_in, scratch, (hipStream_t)stream);
    if (rc) return rc;
    const size_t V = m->cfg.vocab;
    HIP_TRY(launch_softmax_sample(scratch + (size_t)(n_in - 1) * V, (size_t)n_in * V, n_seqs, (int)V, temperature,
                                  u_draft, u_stride, D_row_out, D_stride, token_out, token_stride, (hipStream_t)stream));
    return SPD_OK;
}

int32_t spd_draft_step(spd_model *m, const int32_t *tokens_in, int32_t n_seqs, int32_t n_in, float temperature,
                       const float *u_draft, float *D_row_out, int32_t *token_out, void *stream) {
    if (!m) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_draft_step");
    return spd_draft_step_strided(m, tokens_in, n_in, n_seqs, n_in, temperature, u_draft, 1, D_row_out,
                                  (size_t)m->cfg.vocab, token_out, 1, stream);
}

int32_t spd_accept_workspace_bytes(int32_t n_seqs, int32_t gamma, int32_t vocab, size_t *bytes) {
    if (!bytes || n_seqs < 1 || gamma < 1 || vocab < 1) return fail(SPD_ERR_INVALID_ARG, "bad argument to spd_accept_workspace_bytes");
    *bytes = accept_workspace_bytes(n_seqs, gamma);
    return SPD_OK;
}

int32_t spd_speculative_accept(const float *target, const float *draft, const int32_t *draft_tokens, const float *u,
                               int32_t n_seqs, int32_t gamma, int32_t vocab, float temperature, uint32_t flags,
                               int32_t *n_accepted_out, int32_t *next_token_out, float *accept_prob_out,
                               void *workspace, size_t workspace_bytes, void *stream) {
    if (!target || !draft || !draft_tokens || !u || !n_accepted_out || !next_token_out || !workspace)
        return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_speculative_accept");
    if (n_seqs < 1 || gamma < 1 || gamma > 63 || vocab < 1) return fail(SPD_ERR_INVALID_ARG, "n_seqs, vocab >= 1 and 1 <= gamma <= 63 required");
    if (!(temperature >= 0.f)) return fail(SPD_ERR_INVALID_ARG, "temperature must be >= 0");
    if (flags & ~3u) return fail(SPD_ERR_INVALID_ARG, "unknown flag bits");
    if (workspace_bytes < accept_workspace_bytes(n_seqs, gamma)) return fail(SPD_ERR_CAPACITY, "accept workspace too small");
    AcceptArgs a;
    a.target = target; a.draft = draft; a.draft_tokens = draft_tokens; a.u = u;
    a.n_seqs = n_seqs; a.gamma = gamma; a.vocab = vocab; a.temperature = temperature; a.flags = flags;
    a.n_accepted = n_accepted_out; a.next_token = next_token_out; a.accept_prob = accept_prob_out;
    a.token_stride = gamma;
    a.stats = (float *)workspace;
    HIP_TRY(launch_accept(a, (hipStream_t)stream));
    return SPD_OK;
}

}  // extern "C"

// ---- accept / resample for callers that cannot allocate ----------------------------------------
// The row statistics that spd_speculative_accept keeps in a caller-provided workspace live here in a
// fixed array in device memory.  Every GPU the library runs on holds its own copy at its own address;
// in host code the array's name is only a stand-in for it, so the address is looked up once per
// device (with that device current) and only that pointer is ever handed to a kernel.
namespace {
constexpr size_t kStaticAcceptBytes = 64 * 1024;          // 4096 rows of statistics
static __device__ __align__(256) unsigned char scratch[kStaticAcceptBytes];
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mutex;
void *g_scratch_ptr[kMaxDevices] = {};

int32_t static_scratch(void **out) {
    int dev = -1;
    HIP_TRY(hipGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return fail(SPD_ERR_HIP, "device index %d outside 0..%d", dev, kMaxDevices - 1);
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_ptr[dev]) {
        void *p = nullptr;
        HIP_TRY(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)));
        if (!p) return fail(SPD_ERR_HIP, "hipGetSymbolAddress returned a NULL address");
        g_scratch_ptr[dev] = p;
    }
    *out = g_scratch_ptr[dev];
    return SPD_OK;
}
}  // namespace

extern "C" {

int32_t spd_speculative_accept_static(const float *target, const float *draft, const int32_t *draft_tokens, const float *u,
                                      int32_t n_seqs, int32_t gamma, int32_t vocab, float temperature, uint32_t flags,
                                      int32_t *n_accepted_out, int32_t *next_token_out, float *accept_prob_out, void *stream) {
    if (!target || !draft || !draft_tokens || !u || !n_accepted_out || !next_token_out)
        return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_speculative_accept_static");
    if (n_seqs < 1 || gamma < 1 || gamma > 63 || vocab < 1) return fail(SPD_ERR_INVALID_ARG, "n_seqs, vocab >= 1 and 1 <= gamma <= 63 required");
    if (!(temperature >= 0.f)) return fail(SPD_ERR_INVALID_ARG, "temperature must be >= 0");
    if (flags & ~3u) return fail(SPD_ERR_INVALID_ARG, "unknown flag bits");
    if ((size_t)n_seqs > SPD_STATIC_ACCEPT_MAX_ROWS || accept_workspace_bytes(n_seqs, gamma) > kStaticAcceptBytes)
        return fail(SPD_ERR_CAPACITY, "n_seqs * (2 gamma + 1) = %lld rows exceed the %d rows of the built-in scratch array",
                    (long long)n_seqs * (2 * gamma + 1), SPD_STATIC_ACCEPT_MAX_ROWS);
    void *ws = nullptr;
    int32_t rc = static_scratch(&ws);
    if (rc) return rc;
    AcceptArgs a;
    a.target = target; a.draft = draft; a.draft_tokens = draft_tokens; a.u = u;
    a.n_seqs = n_seqs; a.gamma = gamma; a.vocab = vocab; a.temperature = temperature; a.flags = flags;
    a.n_accepted = n_accepted_out; a.next_token = next_token_out; a.accept_prob = accept_prob_out;
    a.token_stride = gamma;
    a.stats = (float *)ws;            // nothing to clear: entries that this call has not written are not taken for its own (its number marks the answers)
    HIP_TRY(launch_accept(a, (hipStream_t)stream));
    return SPD_OK;
}

int32_t spd_block_finish(spd_model *target, spd_model *draft, const float *target_logits, const float *draft_probs,
                         int32_t *verify_tokens, const float *u, int32_t n_seqs, int32_t gamma, float temperature,
                         int32_t *n_accepted_out, int32_t *next_token_out, int32_t *draft_in_out, int32_t *out_tokens,
                         int32_t out_capacity, int32_t *n_out, void *workspace, size_t workspace_bytes, void *stream) {
    if (!target || !draft || !target_logits || !draft_probs || !verify_tokens || !u || !n_accepted_out || !next_token_out ||
        !draft_in_out || !workspace || (out_tokens && !n_out))
        return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_block_finish");
    if (!target->dev_lens || !draft->dev_lens)
        return fail(SPD_ERR_INVALID_ARG, "spd_block_finish needs both models' KV lengths on the device (spd_kv_lens_to_device)");
    if (n_seqs < 1 || n_seqs > target->cfg.max_seqs || n_seqs > draft->cfg.max_seqs) return fail(SPD_ERR_CAPACITY, "n_seqs exceeds max_seqs");
    if (gamma < 1 || gamma + 1 > SPD_MAX_M) return fail(SPD_ERR_SHAPE, "gamma + 1 must be in 2..%d", SPD_MAX_M);
    if (target->cfg.vocab != draft->cfg.vocab) return fail(SPD_ERR_SHAPE, "target and draft vocabularies differ");
    if (!(temperature >= 0.f)) return fail(SPD_ERR_INVALID_ARG, "temperature must be >= 0");
    if (out_tokens && out_capacity < 1) return fail(SPD_ERR_INVALID_ARG, "out_capacity must be positive");
    if (workspace_bytes < accept_workspace_bytes(n_seqs, gamma)) return fail(SPD_ERR_CAPACITY, "accept workspace too small");
    AcceptArgs a;
    a.target = target_logits; a.draft = draft_probs; a.draft_tokens = verify_tokens + 1; a.token_stride = gamma + 1; a.u = u;
    a.n_seqs = n_seqs; a.gamma = gamma; a.vocab = target->cfg.vocab; a.temperature = temperature; a.flags = SPD_DRAFT_IS_PROBS;
    a.n_accepted = n_accepted_out; a.next_token = next_token_out; a.accept_prob = nullptr;
    a.stats = (float *)workspace;
    HIP_TRY(launch_accept(a, (hipStream_t)stream));
    CommitArgs cm;
    cm.n_accepted = n_accepted_out; cm.next_token = next_token_out; cm.verify_tokens = verify_tokens; cm.draft_in = draft_in_out;
    cm.target_lens = (int32_t *)(target->ws + target->L.d_lens); cm.draft_lens = (int32_t *)(draft->ws + draft->L.d_lens);
    cm.out_tokens = out_tokens; cm.n_out = n_out; cm.n_seqs = n_seqs; cm.gamma = gamma; cm.out_capacity = out_capacity;
    HIP_TRY(launch_block_commit(cm, (hipStream_t)stream));
    // host bounds: at most gamma + 1 positions per sequence were added by the verify call and stay, at least one did
    for (spd_model *m : {target, draft})
        for (int s = 0; s < n_seqs; ++s) m->lens_least[s] = std::min(m->lens_least[s] + 1, m->cfg.max_positions);
    return SPD_OK;
}

}  // extern "C"

// ---- weights in 4 bits -------------------------------------------------------------------------
namespace {
int32_t check_q4(const char *what, int32_t N, int32_t K, int32_t group) {
    if (N < 1 || K < 1) return fail(SPD_ERR_SHAPE, "%s: N = %d and K = %d must be positive", what, N, K);
    if (!q4_group_ok(group)) return fail(SPD_ERR_SHAPE, "%s: group %d must be 32, 64 or 128", what, group);
    // (a launch has fewer than 2^32 threads: a wave per 512 weights of a row; and the digits of a row group are reached by 32-bit offsets)
    if (K > SPD_Q4_MAX_K || (int64_t)N * ((K + 511) / 512) > ((int64_t)1 << 26) - 4) return fail(SPD_ERR_SHAPE, "%s: %d x %d is too large", what, N, K);
    return SPD_OK;
}
constexpr uint32_t kTypeFlags = SPD_W_IS_BF16;
}  // namespace

extern "C" {

int32_t spd_q4_bytes(int32_t N, int32_t K, int32_t group, size_t *bytes) {
    if (!bytes) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_q4_bytes");
    const int32_t rc = check_q4("spd_q4_bytes", N, K, group);
    if (rc) return rc;
    *bytes = q4_packed_bytes(N, K, group);
    return SPD_OK;
}

int32_t spd_q4_quantize(const void *w, size_t w_stride, uint32_t flags, int32_t N, int32_t K, int32_t group, void *q_out, void *scales_out, void *stream) {
    if (!w || !q_out || !scales_out) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_q4_quantize");
    const int32_t rc = check_q4("spd_q4_quantize", N, K, group);
    if (rc) return rc;
    if (flags & ~kTypeFlags) return fail(SPD_ERR_INVALID_ARG, "unknown flag bits");
    if (w_stride < (size_t)K) return fail(SPD_ERR_INVALID_ARG, "w_stride must cover a row");
    HIP_TRY(launch_q4_quantize(w, flags & SPD_W_IS_BF16, w_stride, N, K, group, q_out, scales_out, (hipStream_t)stream));
    return SPD_OK;
}

int32_t spd_q4_dequantize(const void *q, const void *scales, int32_t N, int32_t K, int32_t group, void *w_out, size_t w_stride, uint32_t flags, void *stream) {
    if (!q || !scales || !w_out) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_q4_dequantize");
    const int32_t rc = check_q4("spd_q4_dequantize", N, K, group);
    if (rc) return rc;
    if (flags & ~kTypeFlags) return fail(SPD_ERR_INVALID_ARG, "unknown flag bits");
    if (w_stride < (size_t)K) return fail(SPD_ERR_INVALID_ARG, "w_stride must cover a row");
    HIP_TRY(launch_q4_dequantize(q, scales, N, K, group, w_out, flags & SPD_W_IS_BF16, w_stride, (hipStream_t)stream));
    return SPD_OK;
}

int32_t spd_q4_pack(const void *q, const void *scales, int32_t N, int32_t K, int32_t group, void *packed, size_t packed_bytes, void *stream) {
    if (!q || !scales || !packed) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_q4_pack");
    const int32_t rc = check_q4("spd_q4_pack", N, K, group);
    if (rc) return rc;
    if ((uintptr_t)packed & 255) return fail(SPD_ERR_INVALID_ARG, "packed must be 256-byte aligned");
    if (packed_bytes < q4_packed_bytes(N, K, group)) return fail(SPD_ERR_CAPACITY, "buffer smaller than spd_q4_bytes reports");
    const void *const qs[3] = {q, nullptr, nullptr}, *const ss[3] = {scales, nullptr, nullptr};
    HIP_TRY(launch_q4_pack(qs, ss, PACK_PLAIN, N, K, group, packed, (hipStream_t)stream));
    return SPD_OK;
}

int32_t spd_q4_matmul_workspace_bytes(int32_t rows, int32_t N, int32_t K, size_t *bytes) {
    if (!bytes) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_q4_matmul_workspace_bytes");
    if (rows < 1 || rows > SPD_MAX_ROWS) return fail(SPD_ERR_SHAPE, "rows = %d must be in 1..%d", rows, SPD_MAX_ROWS);
    const int32_t rc = check_q4("spd_q4_matmul_workspace_bytes", N, K, 32);
    if (rc) return rc;
    *bytes = q4_workspace_bytes(rows, N, K);
    return SPD_OK;
}

int32_t spd_q4_matmul(const void *packed, int32_t N, int32_t K, int32_t group, const void *x, size_t x_stride, uint32_t flags, int32_t rows,
                      float *y, size_t y_stride, void *workspace, size_t workspace_bytes, void *stream) {
    if (!packed || !x || !y) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_q4_matmul");
    const int32_t rc = check_q4("spd_q4_matmul", N, K, group);
    if (rc) return rc;
    if (rows < 1 || rows > SPD_MAX_ROWS) return fail(SPD_ERR_SHAPE, "rows = %d must be in 1..%d", rows, SPD_MAX_ROWS);
    if (flags & ~SPD_X_IS_BF16) return fail(SPD_ERR_INVALID_ARG, "unknown flag bits");
    if (x_stride < (size_t)K || y_stride < (size_t)N) return fail(SPD_ERR_INVALID_ARG, "strides must cover a row");
    if (((uintptr_t)packed & 255) || ((uintptr_t)workspace & 255)) return fail(SPD_ERR_INVALID_ARG, "packed and workspace must be 256-byte aligned");
    const size_t need = q4_workspace_bytes(rows, N, K);
    if (need && (!workspace || workspace_bytes < need)) return fail(SPD_ERR_CAPACITY, "workspace smaller than spd_q4_matmul_workspace_bytes reports");
    Q4GemmArgs a{};
    a.W = packed; a.N = N; a.K = K; a.group = group; a.rows = rows;
    a.X = x; a.x_kind = flags & SPD_X_IS_BF16 ? Q4_X_BF16 : Q4_X_F32; a.ldx = x_stride;
    a.Y = y; a.ldy = y_stride;
    a.workspace = workspace;
    HIP_TRY(launch_q4_gemm(a, EPI_STORE, (hipStream_t)stream));
    return SPD_OK;
}

}  // extern "C"

// ---- log probabilities -------------------------------------------------------------------------
namespace {
int32_t check_logprobs(int32_t n_rows, int32_t vocab, int32_t n_top) {
    if (n_rows < 1 || vocab < 1) return fail(SPD_ERR_INVALID_ARG, "n_rows, vocab >= 1 required");
    if (vocab > SPD_MAX_LOGPROB_VOCAB) return fail(SPD_ERR_SHAPE, "vocab %d exceeds %d", vocab, SPD_MAX_LOGPROB_VOCAB);
    if (n_top < 0 || n_top > SPD_MAX_TOP) return fail(SPD_ERR_INVALID_ARG, "n_top = %d must be in 0..%d", n_top, SPD_MAX_TOP);
    if (n_rows > SPD_MAX_LOGPROB_ROWS / logprob_slices(vocab)) return fail(SPD_ERR_SHAPE, "n_rows = %d is too many for vocab = %d", n_rows, vocab);
    return SPD_OK;
}
}  // namespace

extern "C" {

int32_t spd_logprobs_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t n_top, size_t *bytes) {
    if (!bytes) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_logprobs_workspace_bytes");
    const int32_t rc = check_logprobs(n_rows, vocab, n_top);
    if (rc) return rc;
    *bytes = logprobs_workspace_bytes(n_rows, vocab, n_top);
    return SPD_OK;
}

int32_t spd_token_logprobs(const float *rows, size_t row_stride, const int32_t *tokens, int32_t n_rows, int32_t vocab, float temperature, uint32_t flags,
                           float *logprob_out, float *entropy_out, int32_t *rank_out, int32_t n_top, int32_t *top_tokens_out, float *top_logprobs_out,
                           void *workspace, size_t workspace_bytes, void *stream) {
    if (!rows || (!tokens && (logprob_out || rank_out)) || (n_top > 0 && (!top_tokens_out || !top_logprobs_out)))
        return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_token_logprobs");
    const int32_t rc = check_logprobs(n_rows, vocab, n_top);
    if (rc) return rc;
    if (row_stride < (size_t)vocab) return fail(SPD_ERR_INVALID_ARG, "row_stride must cover a row");
    if (flags & ~SPD_ROWS_ARE_PROBS) return fail(SPD_ERR_INVALID_ARG, "unknown flag bits");
    const bool probs = flags & SPD_ROWS_ARE_PROBS;
    if (!probs && !logprob_temperature_ok(temperature)) return fail(SPD_ERR_INVALID_ARG, "temperature must be positive and finite, and at least 4.3e-39");
    if ((uintptr_t)workspace & 15) return fail(SPD_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    const size_t need = logprobs_workspace_bytes(n_rows, vocab, n_top);
    if (need && (!workspace || workspace_bytes < need)) return fail(SPD_ERR_CAPACITY, "workspace smaller than spd_logprobs_workspace_bytes reports");
    if (!logprob_out && !entropy_out && !rank_out && n_top == 0) return SPD_OK;
    LogprobArgs a;
    a.rows = rows; a.row_stride = row_stride; a.tokens = tokens; a.n_rows = n_rows; a.vocab = vocab; a.n_top = n_top;
    a.probs = probs; a.inv_temp = probs ? 1.0f : 1.0f / temperature;
    a.logprob = logprob_out; a.entropy = entropy_out; a.rank = rank_out; a.top_tokens = top_tokens_out; a.top_logprobs = top_logprobs_out;
    a.workspace = workspace;
    HIP_TRY(launch_logprobs(a, (hipStream_t)stream));
    return SPD_OK;
}

}  // extern "C"

// ---- rotary positions, paged cache -------------------------------------------------------------
namespace {
int32_t check_rope(const spd_rope *r, int32_t dim) {
    if (!r->table || (uintptr_t)r->table & 15) return fail(SPD_ERR_INVALID_ARG, "the table of rotary positions must be given, 16-byte aligned");
    if (r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > dim) return fail(SPD_ERR_SHAPE, "rotary_dim = %d must be even, in 2..%d", r->rotary_dim, dim);
    if (r->interleaved != 0 && r->interleaved != 1) return fail(SPD_ERR_INVALID_ARG, "interleaved must be 0 or 1");
    return SPD_OK;
}
// `size`: bytes of an element
int32_t check_heads(const char *what, const spd_heads *h, int32_t n_rows, int32_t n_heads, int32_t dim, size_t size) {
    if (!h->data) return fail(SPD_ERR_INVALID_ARG, "NULL data of %s", what);
    if ((uintptr_t)h->data % size) return fail(SPD_ERR_INVALID_ARG, "data of %s must be aligned to its elements", what);
    const size_t most = (size_t)1 << 40;
    if (h->row_stride > most || h->head_stride > most) return fail(SPD_ERR_INVALID_ARG, "strides of %s are too large", what);
    // heads within rows, or rows within heads
    const size_t in_row = (size_t)(n_heads - 1) * h->head_stride + dim, in_head = (size_t)(n_rows - 1) * h->row_stride + dim;
    const bool apart = (n_heads == 1 || h->head_stride >= (size_t)dim) && (n_rows == 1 || h->row_stride >= (size_t)dim) &&
                       (n_rows == 1 || n_heads == 1 || h->row_stride >= in_row || h->head_stride >= in_head);
    return apart ? SPD_OK : fail(SPD_ERR_INVALID_ARG, "heads of %s overlap", what);
}
HeadsArgs heads_args(const spd_heads *h) { return {h->data, h->row_stride, h->head_stride}; }

int32_t check_paged(const spd_paged_cache *c, const spd_paged_batch *b, PagedCacheArgs &ca, PagedBatchArgs &ba) {
    if (!c || !b || !c->k || !c->v || !b->page_table || !b->lens) return fail(SPD_ERR_INVALID_ARG, "NULL argument to a paged call");
    if (c->head_dim != 64 && c->head_dim != 128) return fail(SPD_ERR_SHAPE, "head_dim = %d must be 64 or 128", c->head_dim);
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return fail(SPD_ERR_SHAPE, "page_size = %d must be 16, 32, 64, 128 or 256", c->page_size);
    if (c->n_pages < 1) return fail(SPD_ERR_SHAPE, "n_pages >= 1 required");
    if (c->n_kv_heads < 1 || c->n_kv_heads > SPD_MAX_PAGED_HEADS) return fail(SPD_ERR_SHAPE, "n_kv_heads = %d must be in 1..%d", c->n_kv_heads, SPD_MAX_PAGED_HEADS);
    if (c->e4m3 != 0 && c->e4m3 != 1) return fail(SPD_ERR_INVALID_ARG, "e4m3 must be 0 or 1");
    if (c->e4m3 ? !c->k_scale || !c->v_scale : c->k_scale || c->v_scale) return fail(SPD_ERR_INVALID_ARG, "scales go with e4m3, both of them");
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return fail(SPD_ERR_INVALID_ARG, "pages must be 16-byte aligned");
    if (b->n_seqs < 1 || b->n_seqs > SPD_MAX_PAGED_SEQS) return fail(SPD_ERR_SHAPE, "n_seqs = %d must be in 1..%d", b->n_seqs, SPD_MAX_PAGED_SEQS);
    if (b->n_rows < 1 || b->n_rows > SPD_MAX_PAGED_ROWS) return fail(SPD_ERR_SHAPE, "n_rows = %d must be in 1..%d", b->n_rows, SPD_MAX_PAGED_ROWS);
    if (b->max_pages < 1 || b->max_pages > SPD_MAX_PAGED_POSITIONS / c->page_size) return fail(SPD_ERR_SHAPE, "max_pages = %d must be in 1..%d", b->max_pages, SPD_MAX_PAGED_POSITIONS / c->page_size);
    if (b->table_stride < (size_t)b->max_pages && b->n_seqs > 1) return fail(SPD_ERR_INVALID_ARG, "table_stride must cover a row of the page table");
    if (b->table_stride > (size_t)1 << 40) return fail(SPD_ERR_INVALID_ARG, "table_stride is too large");
    if (!b->row_start && b->n_rows % b->n_seqs) return fail(SPD_ERR_SHAPE, "without row_start n_rows = %d must be a multiple of n_seqs = %d", b->n_rows, b->n_seqs);
    ca.k = c->k; ca.v = c->v; ca.k_scale = c->k_scale; ca.v_scale = c->v_scale;
    ca.n_pages = c->n_pages; ca.page_bits = __builtin_ctz((unsigned)c->page_size); ca.n_kv = c->n_kv_heads; ca.dim = c->head_dim; ca.e4m3 = c->e4m3;
    ba.n_seqs = b->n_seqs; ba.n_rows = b->n_rows; ba.max_pages = b->max_pages; ba.each = b->n_rows / b->n_seqs; ba.capacity = b->max_pages * c->page_size;
    ba.table_stride = b->table_stride; ba.page_table = b->page_table; ba.lens = b->lens; ba.row_start = b->row_start;
    return SPD_OK;
}
int32_t check_query_heads(int32_t n_heads, int32_t n_kv) {
    if (n_heads < 1 || n_heads > SPD_MAX_PAGED_HEADS || n_heads % n_kv) return fail(SPD_ERR_SHAPE, "n_heads = %d must be a multiple of n_kv_heads = %d, at most %d", n_heads, n_kv, SPD_MAX_PAGED_HEADS);
    return SPD_OK;
}
bool positive(float x) { return x > 0.0f && std::isfinite(x); }
}  // namespace

extern "C" {

int32_t spd_rope_table_bytes(int32_t rotary_dim, size_t *bytes) {
    if (!bytes) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_rope_table_bytes");
    if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > SPD_MAX_HEAD_DIM) return fail(SPD_ERR_SHAPE, "rotary_dim = %d must be even, in 2..%d", rotary_dim, SPD_MAX_HEAD_DIM);
    *bytes = kRopeHeader + (size_t)rotary_dim / 2 * sizeof(uint64_t);
    return SPD_OK;
}

int32_t spd_rope_table(const spd_rope_config *c, void *table, size_t table_bytes, void *stream) {
    if (!c || !table) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_rope_table");
    size_t need;
    const int32_t rc = spd_rope_table_bytes(c->rotary_dim, &need);
    if (rc) return rc;
    if ((uintptr_t)table & 15) return fail(SPD_ERR_INVALID_ARG, "table must be 16-byte aligned");
    if (table_bytes < need) return fail(SPD_ERR_CAPACITY, "table smaller than spd_rope_table_bytes reports");
    if (!positive(c->theta) || !std::isfinite(c->magnitude)) return fail(SPD_ERR_INVALID_ARG, "theta must be positive, theta and magnitude finite");
    if (c->scaling < SPD_ROPE_NONE || c->scaling > SPD_ROPE_LOG_RAMP) return fail(SPD_ERR_INVALID_ARG, "scaling = %d is unknown", c->scaling);
    const bool ramp = c->scaling == SPD_ROPE_RAMP || c->scaling == SPD_ROPE_LOG_RAMP;
    if (c->scaling != SPD_ROPE_NONE && !positive(c->factor)) return fail(SPD_ERR_INVALID_ARG, "factor must be positive and finite");
    if (ramp && (!positive(c->original_positions) || !std::isfinite(c->low) || !std::isfinite(c->high) || !(c->high > c->low) || (c->scaling == SPD_ROPE_LOG_RAMP && !(c->low > 0.0f))))
        return fail(SPD_ERR_INVALID_ARG, "a ramp needs original_positions > 0 and low < high, finite (0 < low where it is one of logarithms)");
    RopeTableArgs a;
    a.n = c->rotary_dim / 2;
    a.magnitude = c->magnitude;
    const long double two_pi = 6.283185307179586476925286766559L;
    for (int i = 0; i < a.n; ++i) {
        if (c->h_factors && !positive(c->h_factors[i])) return fail(SPD_ERR_INVALID_ARG, "h_factors must be positive and finite");
        long double f = powl(c->theta, -2.0L * i / c->rotary_dim) / (c->h_factors ? (long double)c->h_factors[i] : 1.0L);
        if (c->scaling == SPD_ROPE_LINEAR) f /= c->factor;
        if (ramp) {
            const long double t = c->original_positions * f / two_pi;
            const long double at = c->scaling == SPD_ROPE_RAMP ? (t - c->low) / ((long double)c->high - c->low) : (logl(t) - logl(c->low)) / (logl(c->high) - logl(c->low));
            const long double r = std::min(1.0L, std::max(0.0L, at));
            f *= r + (1.0L - r) / c->factor;
        }
        f /= two_pi;
        f -= floorl(f);                                                     // whole turns are none
        a.turn[i] = f > 0.0L ? (uint64_t)std::min(ldexpl(f, 64), ldexpl(1.0L, 64) - 1.0L) : 0;
    }
    HIP_TRY(launch_rope_table(a, table, (hipStream_t)stream));
    return SPD_OK;
}

int32_t spd_rope_apply(const spd_rope *rope, const spd_heads *x, const spd_heads *out, const int32_t *positions, int32_t n_rows, int32_t n_heads,
                       int32_t head_dim, uint32_t flags, void *stream) {
    if (!rope || !x || !out || !positions) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_rope_apply");
    if (n_rows < 1 || n_rows > SPD_MAX_PAGED_ROWS || n_heads < 1 || n_heads > SPD_MAX_PAGED_HEADS || head_dim < 2 || head_dim > SPD_MAX_HEAD_DIM)
        return fail(SPD_ERR_SHAPE, "n_rows in 1..%d, n_heads in 1..%d and head_dim in 2..%d required", SPD_MAX_PAGED_ROWS, SPD_MAX_PAGED_HEADS, SPD_MAX_HEAD_DIM);
    if (flags & ~(SPD_X_IS_BF16 | SPD_ROPE_INVERSE)) return fail(SPD_ERR_INVALID_ARG, "unknown flag bits");
    const size_t size = flags & SPD_X_IS_BF16 ? 2 : 4;
    int32_t rc = check_rope(rope, head_dim);
    if (!rc) rc = check_heads("x", x, n_rows, n_heads, head_dim, size);
    if (!rc) rc = check_heads("out", out, n_rows, n_heads, head_dim, size);
    if (rc) return rc;
    if (x->data == out->data && (x->row_stride != out->row_stride || x->head_stride != out->head_stride)) return fail(SPD_ERR_INVALID_ARG, "out in the place of x has the strides of x");
    RopeArgs a;
    a.x = heads_args(x); a.out = heads_args(out); a.rope = {rope->table, rope->rotary_dim, rope->interleaved != 0};
    a.positions = positions; a.n_rows = n_rows; a.n_heads = n_heads; a.dim = head_dim;
    a.bf16 = flags & SPD_X_IS_BF16; a.inverse = flags & SPD_ROPE_INVERSE;
    HIP_TRY(launch_rope(a, (hipStream_t)stream));
    return SPD_OK;
}

int32_t spd_paged_append(const spd_paged_cache *cache, const spd_paged_batch *batch, const spd_heads *k, const spd_heads *v, const spd_heads *q, const spd_heads *q_out,
                         int32_t n_heads, const spd_rope *rope, const int32_t *positions, uint32_t flags, void *stream) {
    if (!k || !v || !q != !q_out) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_paged_append (q and q_out go together)");
    PagedAppendArgs a{};
    int32_t rc = check_paged(cache, batch, a.c, a.b);
    if (rc) return rc;
    if (flags & ~SPD_X_IS_BF16) return fail(SPD_ERR_INVALID_ARG, "unknown flag bits");
    if (!rope && (q || positions)) return fail(SPD_ERR_INVALID_ARG, "queries and positions go with rotary positions");
    const size_t size = flags & SPD_X_IS_BF16 ? 2 : 4;
    const int rows = batch->n_rows, dim = cache->head_dim;
    rc = check_heads("k", k, rows, cache->n_kv_heads, dim, size);
    if (!rc) rc = check_heads("v", v, rows, cache->n_kv_heads, dim, size);
    if (!rc && rope) rc = check_rope(rope, dim);
    if (!rc && q) {
        if (n_heads < 1 || n_heads > SPD_MAX_PAGED_HEADS) return fail(SPD_ERR_SHAPE, "n_heads = %d must be in 1..%d", n_heads, SPD_MAX_PAGED_HEADS);
        rc = check_heads("q", q, rows, n_heads, dim, size);
        if (!rc) rc = check_heads("q_out", q_out, rows, n_heads, dim, size);
        if (!rc && q->data == q_out->data && (q->row_stride != q_out->row_stride || q->head_stride != q_out->head_stride))
            rc = fail(SPD_ERR_INVALID_ARG, "q_out in the place of q has the strides of q");
    }
    if (rc) return rc;
    if ((int64_t)rows * ((q ? n_heads : 0) + 2 * cache->n_kv_heads) > SPD_MAX_PAGED_ROW_HEADS) return fail(SPD_ERR_SHAPE, "rows times heads of q, k and v exceed %d", SPD_MAX_PAGED_ROW_HEADS);
    a.k = heads_args(k); a.v = heads_args(v);
    if (q) { a.q = heads_args(q); a.q_out = heads_args(q_out); a.n_heads = n_heads; }
    if (rope) a.rope = {rope->table, rope->rotary_dim, rope->interleaved != 0};
    a.positions = positions; a.bf16 = flags & SPD_X_IS_BF16;
    HIP_TRY(launch_paged_append(a, (hipStream_t)stream));
    return SPD_OK;
}

int32_t spd_paged_attention_workspace_bytes(const spd_paged_cache *cache, const spd_paged_batch *batch, int32_t n_heads, size_t *bytes) {
    if (!bytes) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_paged_attention_workspace_bytes");
    PagedCacheArgs c;
    PagedBatchArgs b;
    int32_t rc = check_paged(cache, batch, c, b);
    if (!rc) rc = check_query_heads(n_heads, c.n_kv);
    if (rc) return rc;
    *bytes = paged_attention_workspace_bytes(c, b, n_heads);
    return SPD_OK;
}

int32_t spd_paged_attention(const spd_paged_cache *cache, const spd_paged_batch *batch, const spd_heads *q, const spd_heads *out, int32_t n_heads, float scale,
                            int32_t window, const uint64_t *seen, float *lse_out, uint32_t flags, void *workspace, size_t workspace_bytes, void *stream) {
    if (!q || !out) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_paged_attention");
    PagedAttentionArgs a{};
    int32_t rc = check_paged(cache, batch, a.c, a.b);
    if (!rc) rc = check_query_heads(n_heads, a.c.n_kv);
    if (rc) return rc;
    if (flags & ~SPD_X_IS_BF16) return fail(SPD_ERR_INVALID_ARG, "unknown flag bits");
    const size_t size = flags & SPD_X_IS_BF16 ? 2 : 4;
    rc = check_heads("q", q, a.b.n_rows, n_heads, a.c.dim, size);
    if (!rc) rc = check_heads("out", out, a.b.n_rows, n_heads, a.c.dim, size);
    if (rc) return rc;
    if (q->data == out->data) return fail(SPD_ERR_INVALID_ARG, "out must not overlap q");
    if (!std::isfinite(scale)) return fail(SPD_ERR_INVALID_ARG, "scale must be finite");
    if (window < 0) return fail(SPD_ERR_INVALID_ARG, "window must not be negative");
    if (window && seen) return fail(SPD_ERR_INVALID_ARG, "a window and a tree of rows do not go together");
    const size_t need = paged_attention_workspace_bytes(a.c, a.b, n_heads);
    if ((uintptr_t)workspace & 255) return fail(SPD_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (need && (!workspace || workspace_bytes < need)) return fail(SPD_ERR_CAPACITY, "workspace smaller than spd_paged_attention_workspace_bytes reports");
    a.q = heads_args(q); a.out = heads_args(out); a.n_heads = n_heads; a.window = window; a.scale = scale; a.seen = seen; a.lse = lse_out;
    a.bf16 = flags & SPD_X_IS_BF16; a.workspace = workspace;
    HIP_TRY(launch_paged_attention(a, (hipStream_t)stream));
    return SPD_OK;
}

// what spd_verify_forward_paged needs behind the attention's own workspace
static int32_t check_verify_paged(const spd_model *m, const spd_paged_cache *layers, const spd_paged_batch *batch, PagedCacheArgs &c, PagedBatchArgs &b) {
    if (!m || !layers) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_verify_forward_paged");
    for (int l = 0; l < m->cfg.n_layers; ++l) {
        const int32_t rc = check_paged(layers + l, batch, c, b);
        if (rc) return rc;
        if (c.n_kv != m->cfg.n_heads || c.dim != m->cfg.head_dim) return fail(SPD_ERR_SHAPE, "pages of layer %d have %d heads of %d, the model %d of %d", l, c.n_kv, c.dim, m->cfg.n_heads, m->cfg.head_dim);
        if (layers[l].page_size != layers[0].page_size || layers[l].n_pages != layers[0].n_pages || layers[l].e4m3 != layers[0].e4m3) return fail(SPD_ERR_SHAPE, "the layers' pages differ");
    }
    if (b.n_rows > SPD_MAX_ROWS) return fail(SPD_ERR_SHAPE, "n_rows = %d must be in 1..%d", b.n_rows, SPD_MAX_ROWS);
    return SPD_OK;
}

int32_t spd_verify_paged_workspace_bytes(const spd_model *m, const spd_paged_cache *layers, const spd_paged_batch *batch, size_t *bytes) {
    if (!bytes) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_verify_paged_workspace_bytes");
    PagedCacheArgs c;
    PagedBatchArgs b;
    const int32_t rc = check_verify_paged(m, layers, batch, c, b);
    if (rc) return rc;
    *bytes = align_up(paged_attention_workspace_bytes(c, b, m->cfg.n_heads), 256) + (size_t)b.n_rows * c.n_kv * c.dim * sizeof(float);
    return SPD_OK;
}

int32_t spd_verify_forward_paged(spd_model *m, const int32_t *tokens, const spd_paged_cache *layers, const spd_paged_batch *batch, const spd_rope *rope, const int32_t *positions,
                                 const uint64_t *seen, float *logits_out, void *workspace, size_t workspace_bytes, void *stream) {
    if (!tokens || !rope || !logits_out) return fail(SPD_ERR_INVALID_ARG, "NULL argument to spd_verify_forward_paged");
    if (seen && !positions) return fail(SPD_ERR_INVALID_ARG, "a tree of rows needs positions: its branches share them, which the rows' own do not say");
    PagedLayers pages{};
    PagedAppendArgs &ap = pages.append;
    PagedAttentionArgs &pa = pages.attention;
    int32_t rc = check_verify_paged(m, layers, batch, ap.c, ap.b);
    if (!rc) rc = check_rope(rope, ap.c.dim);
    if (rc) return rc;
    const spd_model_config &c = m->cfg;
    const Layout &L = m->L;
    const int rows = ap.b.n_rows, dim = c.head_dim, HD = c.n_heads * dim;
    const size_t attention_bytes = align_up(paged_attention_workspace_bytes(ap.c, ap.b, c.n_heads), 256);
    if ((uintptr_t)workspace & 255) return fail(SPD_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (!workspace || workspace_bytes < attention_bytes + (size_t)rows * HD * sizeof(float)) return fail(SPD_ERR_CAPACITY, "workspace smaller than spd_verify_paged_workspace_bytes reports");
    float *qkv = (float *)(m->ws + L.qkv);
    pages.cache = layers;
    pages.rows = (float *)((char *)workspace + attention_bytes);
    auto heads = [&](float *p) { return HeadsArgs{p, (size_t)3 * HD, (size_t)dim}; };
    ap.q = ap.q_out = heads(qkv); ap.k = heads(qkv + HD); ap.v = heads(qkv + 2 * HD);
    ap.n_heads = c.n_heads; ap.rope = {rope->table, rope->rotary_dim, rope->interleaved != 0}; ap.positions = positions; ap.bf16 = false;
    pa.c = ap.c; pa.b = ap.b; pa.q = ap.q_out; pa.out = {pages.rows, (size_t)HD, (size_t)dim};
    pa.n_heads = c.n_heads; pa.window = 0; pa.scale = 1.0f / sqrtf((float)dim); pa.seen = seen; pa.lse = nullptr; pa.bf16 = false; pa.workspace = workspace;
    hipStream_t st = (hipStream_t)stream;
    // rows behind the last sequence have no attention: zeros, so that what follows works on numbers
    if (ap.b.row_start) HIP_TRY(launch_fill_zero(pages.rows, (size_t)rows * HD * sizeof(float), st));
    PROF_TRY(PK_EMBED, launch_input_rows(m->packed + L.embed, tokens, rows, rows, nullptr, rows, c.d_model, c.vocab, (const float *)(m->packed + L.attn_norm[0]),
                                         (float *)(m->ws + L.h), m->ws + L.xn, (float *)(m->ws + L.ssq_b), st));
    AttnArgs at{};
    return run_layers(m, 0, at, 0, 1, rows, 0, false, logits_out, st, &pages);
}

}  // extern "C"
