// C ABI of the training operators: argument validation and launches.
#include <hip/hip_runtime.h>
#include <cmath>
#include <initializer_list>
#include "../../include/pipedit_train.h"
#include "attn_internal.h"
#include "train_internal.h"

namespace {

using pda::report;

int hip_error(hipError_t e, const char* what) { return report(PDA_ERR_HIP, "%s: %s", what, hipGetErrorString(e)); }

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool bad_type(int t) { return t != PDA_F32 && t != PDA_BF16; }

// Do the ranges [a, a + na) and [b, b + nb) share a byte?
bool overlap(const void* a, double na, const void* b, double nb) {
    const double x = (double)reinterpret_cast<uintptr_t>(a), y = (double)reinterpret_cast<uintptr_t>(b);
    return na > 0 && nb > 0 && x < y + nb && y < x + na;
}

struct Range {
    const void* p;           // null: not there
    double bytes;
    const char* name;
};
int check_apart(std::initializer_list<Range> written, std::initializer_list<Range> others) {
    for (const Range& w : written)
        for (const Range& x : others)
            if (w.p && x.p && overlap(w.p, w.bytes, x.p, x.bytes)) return report(PDA_ERR_INVALID_ARG, "%s overlaps %s", w.name, x.name);
    return PDA_OK;
}

int check_bwd_sizes(int B, int H, int64_t Sq, int64_t Skv, int d, int64_t kv_valid_len) {
    if (B < 0 || H < 0 || Sq < 0 || Skv < 0) return report(PDA_ERR_INVALID_ARG, "negative size (B=%d H=%d Sq=%lld Skv=%lld)", B, H, (long long)Sq, (long long)Skv);
    if (d != 64 && d != 128) return report(PDA_ERR_UNSUPPORTED, "head dim d=%d not supported (64 or 128)", d);
    if (kv_valid_len < 0 || kv_valid_len > Skv) return report(PDA_ERR_INVALID_ARG, "kv_valid_len=%lld outside [0, Skv=%lld]", (long long)kv_valid_len, (long long)Skv);
    if (Sq >= (int64_t)1 << 31 || Skv >= (int64_t)1 << 31) return report(PDA_ERR_UNSUPPORTED, "sequence length beyond 2^31");
    if ((double)B * H * (double)(Sq > Skv ? Sq : Skv) * d >= 1099511627776.0) return report(PDA_ERR_UNSUPPORTED, "B*H*S*d overflows 2^40 elements");
    if ((int64_t)B * H > 65535) return report(PDA_ERR_UNSUPPORTED, "B*H > 65535");
    return PDA_OK;
}

// B x H blocks of `bytes` bytes, `batch` and `head` bytes apart.
struct View {
    const void* p;           // null: not there
    int64_t bytes, B, H, batch, head;
    const char* name;
    int64_t span() const { return (B - 1) * batch + (H - 1) * head + bytes; }
};
View view(const void* p, int64_t n, int size, int B, int H, int64_t batch, int64_t head, const char* name) {
    View v{p, n * size, B, H, batch * size, head * size, name};
    if (v.head == v.bytes || H == 1) v = View{p, v.bytes * H, B, 1, v.batch, 0, name};       // one piece a batch, or one in all
    if (v.H == 1 && v.batch == v.bytes) v = View{p, v.bytes * B, 1, 1, 0, 0, name};
    return v;
}
// Do two views share a byte?  Every block of one against the blocks of the other that its place leaves.
bool overlap(const View& x, const View& y) {
    if (!x.p || !y.p || x.bytes == 0 || y.bytes == 0) return false;
    const int64_t from = (int64_t)(reinterpret_cast<uintptr_t>(x.p) - reinterpret_cast<uintptr_t>(y.p));
    if (from >= y.span() || from + x.span() <= 0) return false;
    const bool heads_out = y.head > y.batch;                   // the outer axis of y is the one of the larger stride
    const int64_t n1 = heads_out ? y.H : y.B, s1 = heads_out ? y.head : y.batch, n2 = heads_out ? y.B : y.H, s2 = heads_out ? y.batch : y.head;
    const int64_t span2 = (n2 - 1) * s2 + y.bytes;
    // first of the places i * s whose `len` bytes end behind `at`
    const auto first = [](int64_t at, int64_t len, int64_t s) -> int64_t { return at < len ? 0 : s == 0 ? INT64_MAX : (at - len) / s + 1; };
    for (int64_t b = 0; b < x.B; ++b)
        for (int64_t h = 0; h < x.H; ++h) {
            const int64_t at = from + b * x.batch + h * x.head, end = at + x.bytes;
            for (int64_t i = first(at, span2, s1); i < n1 && i * s1 < end; ++i) {
                const int64_t j = first(at - i * s1, y.bytes, s2);
                if (j < n2 && j * s2 < end - i * s1) return true;
                if (s1 == 0) break;
            }
        }
    return false;
}
int check_apart(std::initializer_list<View> written, std::initializer_list<View> others) {
    for (const View& w : written)
        for (const View& x : others)
            if (overlap(w, x)) return report(PDA_ERR_INVALID_ARG, "%s overlaps %s", w.name, x.name);
    return PDA_OK;
}

// The blocks of n elements at b * batch + h * head must not share any, whichever of the two axes is the outer one.
int check_blocks(int B, int H, int64_t batch, int64_t head, int64_t n, const char* name) {
    if (n == 0 || B == 0 || H == 0) return PDA_OK;
    if (H > 1 && head < n) return report(PDA_ERR_INVALID_ARG, "heads of %s overlap (head stride too small)", name);
    for (int64_t i = 1; i < B; ++i) {                          // block (0, h) against (i, 0); differences with h on the other side are larger
        const int64_t x = i * batch;
        if (x >= (H - 1) * head + n) break;
        int64_t h = H > 1 ? x / head : 0;                      // the nearest ones
        h = h < H - 1 ? h : H - 1;
        if (x - h * head < n || (h + 1 < H && (h + 1) * head - x < n))
            return report(PDA_ERR_INVALID_ARG, "batches of %s overlap (batch stride %lld, head stride %lld)", name, (long long)batch, (long long)head);
    }
    return PDA_OK;
}

int attn_bwd(const void* dout, const void* q, const void* k, const void* v, const void* out, int out_type, const float* lse,
             void* dq, void* dk, void* dv, int B, int H, int64_t Sq, int64_t Skv, int d, const pda_attn_bwd_strides& s,
             float scale, int64_t n_v, void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_bwd_sizes(B, H, Sq, Skv, d, n_v);
    if (rc != PDA_OK) return rc;
    if (!(scale >= 0.0f) || !std::isfinite(scale)) return report(PDA_ERR_INVALID_ARG, "scale must be finite and >= 0");
    if (bad_type(out_type)) return report(PDA_ERR_INVALID_ARG, "unknown out_type=%d", out_type);
    if (B == 0 || H == 0 || (Sq == 0 && Skv == 0)) return PDA_OK;
    if (Sq > 0 && (!dout || !q || !out || !lse || !dq)) return report(PDA_ERR_INVALID_ARG, "null dout/q/out/lse/dq");
    if (Sq > 0 && n_v > 0 && (!k || !v)) return report(PDA_ERR_INVALID_ARG, "null k/v");
    if (Skv > 0 && (!dk || !dv)) return report(PDA_ERR_INVALID_ARG, "null dk/dv");
    for (const void* p : {dout, q, k, v, out, static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(dv)})
        if (!aligned(p, 16)) return report(PDA_ERR_UNSUPPORTED, "dout/q/k/v/out/dq/dk/dv must be 16-byte aligned");
    if (!aligned(lse, 4)) return report(PDA_ERR_UNSUPPORTED, "lse must be 4-byte aligned");
    const int64_t nq = Sq * d, nk = Skv * d;
    const View rq = view(dq, nq, 2, B, H, s.dq_batch, s.dq_head, "dq"), rk = view(dk, nk, 2, B, H, s.dkv_batch, s.dkv_head, "dk"),
               rv = view(dv, nk, 2, B, H, s.dkv_batch, s.dkv_head, "dv");
    const std::initializer_list<View> in = {
        view(dout, nq, 2, B, H, s.dout_batch, s.dout_head, "dout"), view(q, nq, 2, B, H, s.q_batch, s.q_head, "q"),
        view(out, nq, out_type == PDA_BF16 ? 2 : 4, B, H, s.out_batch, s.out_head, "out"), view(lse, Sq, 4, B, H, s.lse_batch, s.lse_head, "lse"),
        view(k, nk, 2, B, H, s.kv_batch, s.kv_head, "k"), view(v, nk, 2, B, H, s.kv_batch, s.kv_head, "v")};
    if ((rc = check_apart({rq, rk, rv}, in)) != PDA_OK) return rc;
    if ((rc = check_apart({rk}, {rq})) != PDA_OK || (rc = check_apart({rv}, {rq, rk})) != PDA_OK) return rc;
    pda::AttnBwdParams p{};
    const int64_t stat_bytes = pda::bwd_stat_bytes((int64_t)B * H, Sq, d), given = workspace ? workspace_bytes : 0;
    if (given < stat_bytes) return report(PDA_ERR_INVALID_ARG, "workspace of %lld bytes, at least %lld needed", (long long)given, (long long)stat_bytes);
    if (!aligned(workspace, 256)) return report(PDA_ERR_UNSUPPORTED, "workspace must be 256-byte aligned");
    const View ws = view(workspace, given < (int64_t)1 << 60 ? given : (int64_t)1 << 60, 1, 1, 1, 0, 0, "workspace");     // (sums of addresses stay in 64 bits)
    if ((rc = check_apart({ws}, in)) != PDA_OK || (rc = check_apart({ws}, {rq, rk, rv})) != PDA_OK) return rc;
    int n_cu = 0;
    hipError_t e = pda::device_cu_count(&n_cu);
    if (e != hipSuccess) return hip_error(e, "device query");
    p.plan = pda::plan_bwd(Sq, n_v, (int64_t)B * H, d, n_cu);
    const int64_t need = pda::bwd_workspace_bytes(p.plan, (int64_t)B * H, Sq, d);
    if (given < need) return report(PDA_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed for kv_valid_len=%lld (PDA_ANY_LEN: a size for all lengths)", (long long)given, (long long)need, (long long)n_v);
    p.dout = static_cast<const __bf16*>(dout);
    p.q = static_cast<const __bf16*>(q);
    p.k = static_cast<const __bf16*>(k);
    p.v = static_cast<const __bf16*>(v);
    p.out = out;
    p.lse = lse;
    p.dq = static_cast<__bf16*>(dq);
    p.dk = static_cast<__bf16*>(dk);
    p.dv = static_cast<__bf16*>(dv);
    p.Sq = Sq; p.Skv = Skv; p.n_v = n_v;
    p.stat_rows = pda::bwd_stat_rows(Sq);
    p.counter = static_cast<int*>(workspace);
    p.stats = static_cast<float*>(workspace) + pda::kBwdCounterBytes / 4;
    p.parts = static_cast<float*>(workspace) + stat_bytes / 4;
    p.n_cu = n_cu;
    p.do_bs = s.dout_batch; p.do_hs = s.dout_head;
    p.q_bs = s.q_batch; p.q_hs = s.q_head;
    p.kv_bs = s.kv_batch; p.kv_hs = s.kv_head;
    p.o_bs = s.out_batch; p.o_hs = s.out_head;
    p.l_bs = s.lse_batch; p.l_hs = s.lse_head;
    p.dq_bs = s.dq_batch; p.dq_hs = s.dq_head;
    p.dkv_bs = s.dkv_batch; p.dkv_hs = s.dkv_head;
    p.B = B; p.H = H;
    p.out_bf16 = out_type == PDA_BF16 ? 1 : 0;
    p.scale = scale;
    p.scale_log2e = (float)((double)scale * 1.4426950408889634);     // exactly 1 for scale = (float)ln 2
    e = pda::launch_attn_bwd(p, d, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)PDA_OK : hip_error(e, "attention gradient launch");
}

int check_layer_norm(int x_type, int y_type, int64_t rows, int64_t groups, int D) {
    if (bad_type(x_type) || bad_type(y_type)) return report(PDA_ERR_INVALID_ARG, "unknown type (x_type=%d y_type=%d)", x_type, y_type);
    if (rows < 0 || groups < 1) return report(PDA_ERR_INVALID_ARG, "rows=%lld groups=%lld (need >= 0, >= 1)", (long long)rows, (long long)groups);
    if (rows % groups != 0) return report(PDA_ERR_INVALID_ARG, "rows=%lld is not a multiple of groups=%lld", (long long)rows, (long long)groups);
    if (D < 1) return report(PDA_ERR_INVALID_ARG, "D=%d (need >= 1)", D);
    if (D > PDA_LAYER_NORM_MAX) return report(PDA_ERR_UNSUPPORTED, "D=%d exceeds PDA_LAYER_NORM_MAX=%d", D, PDA_LAYER_NORM_MAX);
    if (groups > 65535) return report(PDA_ERR_UNSUPPORTED, "groups=%lld beyond 65535", (long long)groups);
    if (rows >= (int64_t)1 << 31 || (double)rows * D >= 1099511627776.0) return report(PDA_ERR_UNSUPPORTED, "rows beyond 2^31 or rows*D beyond 2^40 elements");
    return PDA_OK;
}

double row_bytes(int64_t rows, int D, int type) { return (double)rows * D * (type == PDA_BF16 ? 2 : 4); }

// An output may be an input itself (equal address and type), but not lie across it.
int check_in_place(const void* out, int out_type, const char* out_name, const void* in, int in_type, const char* in_name, int64_t rows, int D) {
    if (out == in && out_type == in_type) return PDA_OK;
    if (overlap(out, row_bytes(rows, D, out_type), in, row_bytes(rows, D, in_type)))
        return report(PDA_ERR_INVALID_ARG, "%s overlaps %s without being it", out_name, in_name);
    return PDA_OK;
}

}  // namespace

extern "C" {

int pda_attn_bwd_workspace(int B, int H, int64_t Sq, int64_t Skv, int d, int64_t kv_valid_len, int n_cu, int64_t* bytes) {
    const bool any = kv_valid_len == PDA_ANY_LEN;
    int rc = check_bwd_sizes(B, H, Sq, Skv, d, any ? Skv : kv_valid_len);
    if (rc != PDA_OK) return rc;
    if (n_cu < 0) return report(PDA_ERR_INVALID_ARG, "n_cu=%d is negative", n_cu);
    if (!bytes) return report(PDA_ERR_INVALID_ARG, "null bytes");
    if (B == 0 || H == 0) {
        *bytes = 0;
        return PDA_OK;
    }
    if (n_cu == 0) {
        const hipError_t e = pda::device_cu_count(&n_cu);
        if (e != hipSuccess) return hip_error(e, "device query");
    }
    const int64_t BH = (int64_t)B * H;
    *bytes = any ? pda::bwd_workspace_bound(BH, Sq, Skv, d, n_cu) : pda::bwd_workspace_bytes(pda::plan_bwd(Sq, kv_valid_len, BH, d, n_cu), BH, Sq, d);
    return PDA_OK;
}

int pda_attn_bwd(const void* dout, const void* q, const void* k, const void* v, const void* out, int out_type,
                 const float* lse, void* dq, void* dk, void* dv,
                 int B, int H, int64_t Sq, int64_t Skv, int d, float scale, int64_t kv_valid_len,
                 void* workspace, int64_t workspace_bytes, void* stream) {
    const int rc = check_bwd_sizes(B, H, Sq, Skv, d, kv_valid_len);       // before they are multiplied
    if (rc != PDA_OK) return rc;
    const int64_t qh = Sq * d, kh = Skv * d, qb = H * qh, kb = H * kh;
    const pda_attn_bwd_strides s{qb, qh, qb, qh, kb, kh, qb, qh, H * Sq, Sq, qb, qh, kb, kh};
    return attn_bwd(dout, q, k, v, out, out_type, lse, dq, dk, dv, B, H, Sq, Skv, d, s, scale, kv_valid_len, workspace, workspace_bytes, stream);
}

int pda_attn_bwd_strided(const void* dout, const void* q, const void* k, const void* v, const void* out, int out_type,
                         const float* lse, void* dq, void* dk, void* dv,
                         int B, int H, int64_t Sq, int64_t Skv, int d, const pda_attn_bwd_strides* strides, float scale,
                         int64_t kv_valid_len, void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_bwd_sizes(B, H, Sq, Skv, d, kv_valid_len);
    if (rc != PDA_OK) return rc;
    if (!strides) return report(PDA_ERR_INVALID_ARG, "null strides");
    if (bad_type(out_type)) return report(PDA_ERR_INVALID_ARG, "unknown out_type=%d", out_type);
    const pda_attn_bwd_strides& s = *strides;
    for (int64_t x : {s.dout_batch, s.dout_head, s.q_batch, s.q_head, s.kv_batch, s.kv_head, s.out_batch, s.out_head, s.lse_batch, s.lse_head,
                      s.dq_batch, s.dq_head, s.dkv_batch, s.dkv_head})
        if (x < 0 || x >= ((int64_t)1 << 40)) return report(PDA_ERR_INVALID_ARG, "stride %lld outside [0, 2^40)", (long long)x);
    if ((s.dout_batch | s.dout_head | s.q_batch | s.q_head | s.kv_batch | s.kv_head | s.dq_batch | s.dq_head | s.dkv_batch | s.dkv_head) % 8 != 0)
        return report(PDA_ERR_UNSUPPORTED, "strides of bf16 tensors must be multiples of 8 elements");
    if ((s.out_batch | s.out_head) % (out_type == PDA_BF16 ? 8 : 4) != 0) return report(PDA_ERR_UNSUPPORTED, "out strides must be multiples of 16 bytes");
    if ((rc = check_blocks(B, H, s.dq_batch, s.dq_head, Sq * d, "dq")) != PDA_OK || (rc = check_blocks(B, H, s.dkv_batch, s.dkv_head, Skv * d, "dk/dv")) != PDA_OK) return rc;
    return attn_bwd(dout, q, k, v, out, out_type, lse, dq, dk, dv, B, H, Sq, Skv, d, s, scale, kv_valid_len, workspace, workspace_bytes, stream);
}

int pda_layer_norm_fwd(const void* x, int x_type, const float* weight, const float* bias, void* y, int y_type,
                       float* mean, float* rstd, int64_t rows, int64_t groups, int D, float eps, void* stream) {
    int rc = check_layer_norm(x_type, y_type, rows, groups, D);
    if (rc != PDA_OK) return rc;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return report(PDA_ERR_INVALID_ARG, "eps must be finite and >= 0");
    if (!mean != !rstd) return report(PDA_ERR_INVALID_ARG, "mean and rstd go together");
    if (rows == 0) return PDA_OK;
    if (!x || !y) return report(PDA_ERR_INVALID_ARG, "null x/y");
    if (!aligned(x, 16) || !aligned(y, 16) || !aligned(weight, 16) || !aligned(bias, 16)) return report(PDA_ERR_UNSUPPORTED, "x/y/weight/bias must be 16-byte aligned");
    if (!aligned(mean, 4) || !aligned(rstd, 4)) return report(PDA_ERR_UNSUPPORTED, "mean/rstd must be 4-byte aligned");
    if ((rc = check_in_place(y, y_type, "y", x, x_type, "x", rows, D)) != PDA_OK) return rc;
    const double param = (double)groups * D * 4, stat = (double)rows * 4;
    const Range ry{y, row_bytes(rows, D, y_type), "y"}, rm{mean, stat, "mean"}, rr{rstd, stat, "rstd"}, rw{weight, param, "weight"}, rb{bias, param, "bias"};
    if ((rc = check_apart({ry, rm, rr}, {rw, rb})) != PDA_OK) return rc;
    if ((rc = check_apart({rm, rr}, {ry, {x, row_bytes(rows, D, x_type), "x"}})) != PDA_OK || (rc = check_apart({rm}, {rr})) != PDA_OK) return rc;
    pda::LayerNormParams p{};
    p.x = x; p.weight = weight; p.bias = bias; p.y = y; p.mean = mean; p.rstd = rstd;
    p.rows = rows; p.groups = groups; p.group_rows = rows / groups; p.D = D; p.eps = eps;
    const hipError_t e = pda::launch_layer_norm_fwd(p, x_type == PDA_BF16, y_type == PDA_BF16, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)PDA_OK : hip_error(e, "layer norm launch");
}

int pda_layer_norm_bwd_workspace(int64_t rows, int64_t groups, int D, int n_cu, int64_t* bytes) {
    int rc = check_layer_norm(PDA_F32, PDA_F32, rows, groups, D);
    if (rc != PDA_OK) return rc;
    if (n_cu < 0) return report(PDA_ERR_INVALID_ARG, "n_cu=%d is negative", n_cu);
    if (!bytes) return report(PDA_ERR_INVALID_ARG, "null bytes");
    if (n_cu == 0) {
        const hipError_t e = pda::device_cu_count(&n_cu);
        if (e != hipSuccess) return hip_error(e, "device query");
    }
    *bytes = pda::ln_workspace_bytes(rows, groups, D, n_cu);
    return PDA_OK;
}

int pda_layer_norm_bwd(const void* dy, int y_type, const void* x, int x_type, const float* weight, const float* mean,
                       const float* rstd, void* dx, float* dweight, float* dbias, int64_t rows, int64_t groups, int D,
                       void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_layer_norm(x_type, y_type, rows, groups, D);
    if (rc != PDA_OK) return rc;
    if (!dx && !dweight && !dbias) return report(PDA_ERR_INVALID_ARG, "null dx, dweight and dbias: nothing to compute");
    if (!aligned(weight, 16) || !aligned(dweight, 16) || !aligned(dbias, 16)) return report(PDA_ERR_UNSUPPORTED, "weight/dweight/dbias must be 16-byte aligned");
    if (rows == 0 && !dweight && !dbias) return PDA_OK;
    pda::LayerNormParams p{};
    if (rows > 0) {
        if (!dy || !x || !mean || !rstd) return report(PDA_ERR_INVALID_ARG, "null dy/x/mean/rstd");
        if (!aligned(dy, 16) || !aligned(x, 16) || !aligned(dx, 16)) return report(PDA_ERR_UNSUPPORTED, "dy/x/dx must be 16-byte aligned");
        if (!aligned(mean, 4) || !aligned(rstd, 4)) return report(PDA_ERR_UNSUPPORTED, "mean/rstd must be 4-byte aligned");
        if (dx && (rc = check_in_place(dx, x_type, "dx", x, x_type, "x", rows, D)) != PDA_OK) return rc;
        if (dx && (rc = check_in_place(dx, x_type, "dx", dy, y_type, "dy", rows, D)) != PDA_OK) return rc;
        const double param = (double)groups * D * 4, stat = (double)rows * 4;
        const Range rx{x, row_bytes(rows, D, x_type), "x"}, ry{dy, row_bytes(rows, D, y_type), "dy"}, rd{dx, rx.bytes, "dx"}, rw{dweight, param, "dweight"}, rb{dbias, param, "dbias"};
        const std::initializer_list<Range> in = {{weight, param, "weight"}, {mean, stat, "mean"}, {rstd, stat, "rstd"}};
        if ((rc = check_apart({rd, rw, rb}, in)) != PDA_OK || (rc = check_apart({rw, rb}, {rx, ry, rd})) != PDA_OK || (rc = check_apart({rb}, {rw})) != PDA_OK) return rc;
        int n_cu = 0;
        const hipError_t e = pda::device_cu_count(&n_cu);
        if (e != hipSuccess) return hip_error(e, "device query");
        const int64_t need = dweight || dbias ? pda::ln_workspace_bytes(rows, groups, D, n_cu) : 0;
        if (need > 0 && (!workspace || workspace_bytes < need))
            return report(PDA_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed", workspace ? (long long)workspace_bytes : 0LL, (long long)need);
        if (need > 0 && !aligned(workspace, 16)) return report(PDA_ERR_UNSUPPORTED, "workspace must be 16-byte aligned");
        const Range ws{need > 0 ? workspace : nullptr, (double)need, "workspace"};
        if ((rc = check_apart({ws}, in)) != PDA_OK || (rc = check_apart({ws}, {rx, ry, rd, rw, rb})) != PDA_OK) return rc;
        p.group_rows = rows / groups;
        p.chunks = pda::ln_chunks(p.group_rows, groups, D, n_cu);
    }
    p.x = x; p.dy = dy; p.weight = weight; p.y = dx;
    p.mean = const_cast<float*>(mean); p.rstd = const_cast<float*>(rstd);
    p.dweight = dweight; p.dbias = dbias; p.part = static_cast<float*>(workspace);
    p.rows = rows; p.groups = groups; p.D = D;
    const hipError_t e = pda::launch_layer_norm_bwd(p, x_type == PDA_BF16, y_type == PDA_BF16, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)PDA_OK : hip_error(e, "layer norm gradient launch");
}

int pda_pack_heads_bwd(const void* dy, const float* x, float* dx, int B, int64_t S, int H, int d, int unit_rms, float premul, void* stream) {
    if (B < 0 || H < 0 || S < 0) return report(PDA_ERR_INVALID_ARG, "negative size (B=%d H=%d S=%lld)", B, H, (long long)S);
    if (d != 64 && d != 128) return report(PDA_ERR_UNSUPPORTED, "head dim d=%d not supported (64 or 128)", d);
    if ((double)B * H * (double)S * d >= 1099511627776.0) return report(PDA_ERR_UNSUPPORTED, "B*H*S*d overflows 2^40 elements");
    if (H >= 1 << 24) return report(PDA_ERR_UNSUPPORTED, "H=%d heads (fewer than 2^24 supported)", H);       // 256 threads each along one axis
    if (B == 0 || H == 0 || S == 0) return PDA_OK;
    if (!dy || !dx || (unit_rms && !x)) return report(PDA_ERR_INVALID_ARG, "null dy/dx, or x with unit_rms");
    if (!aligned(dy, 16) || !aligned(x, 16) || !aligned(dx, 16)) return report(PDA_ERR_UNSUPPORTED, "dy, x and dx must be 16-byte aligned");
    const double n = (double)B * H * (double)S * d;
    if (overlap(dx, n * 4, dy, n * 2)) return report(PDA_ERR_INVALID_ARG, "dx overlaps dy");
    if (unit_rms && dx != x && overlap(dx, n * 4, x, n * 4)) return report(PDA_ERR_INVALID_ARG, "dx overlaps x without being it");
    if (!std::isfinite(premul)) return report(PDA_ERR_INVALID_ARG, "premul must be finite");
    const hipError_t e = pda::launch_pack_bwd(dy, x, dx, B, S, H, d, unit_rms, premul, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)PDA_OK : hip_error(e, "pack gradient launch");
}

}  // extern "C"
