// C ABI of the projection side: argument validation and launches.
#include <hip/hip_runtime.h>
#include <cmath>
#include "../../include/pipedit_proj.h"
#include "api_checks.h"
#include "attn_internal.h"
#include "proj_internal.h"

namespace {

using namespace pda;

constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr double kMaxElements = 1099511627776.0;         // 2^40

bool bad_fp8(int t) { return t != PDA_E4M3 && t != PDA_E5M2; }
int type_size(int t) { return t == PDA_F32 ? 4 : t == PDA_BF16 ? 2 : 1; }

// ---- norm
int check_rms(int64_t rows, int64_t groups, int D) {
    if (rows < 0 || groups < 1) return report(PDA_ERR_INVALID_ARG, "rows=%lld groups=%lld (need >= 0, >= 1)", (long long)rows, (long long)groups);
    if (rows % groups != 0) return report(PDA_ERR_INVALID_ARG, "rows=%lld is not a multiple of groups=%lld", (long long)rows, (long long)groups);
    if (D < 1) return report(PDA_ERR_INVALID_ARG, "D=%d (need >= 1)", D);
    if (D > PDA_LAYER_NORM_MAX) return report(PDA_ERR_UNSUPPORTED, "D=%d exceeds PDA_LAYER_NORM_MAX=%d", D, PDA_LAYER_NORM_MAX);
    if (groups > 65535) return report(PDA_ERR_UNSUPPORTED, "groups=%lld beyond 65535", (long long)groups);
    if (rows >= kMaxRows || (double)rows * D >= kMaxElements) return report(PDA_ERR_UNSUPPORTED, "rows beyond 2^31 or rows*D beyond 2^40 elements");
    return PDA_OK;
}

// A written tensor may be an input itself (equal address and type), but not lie across it.
int check_itself(const Range& out, int out_type, const Range& in, int in_type) {
    if (out.p && out.p == in.p && out_type == in_type) return PDA_OK;
    return check_apart({out}, {in});
}

// ---- product
int check_matmul(int64_t M, int64_t N, int64_t K) {
    if (M < 0 || N < 0 || K < 0) return report(PDA_ERR_INVALID_ARG, "negative size (M=%lld N=%lld K=%lld)", (long long)M, (long long)N, (long long)K);
    if (K % 128 != 0) return report(PDA_ERR_INVALID_ARG, "K=%lld is not a multiple of 128 (rows are padded to whole blocks)", (long long)K);
    if (M >= kMaxRows || N >= kMaxRows || K >= 1 << 24) return report(PDA_ERR_UNSUPPORTED, "M or N beyond 2^31, or K=%lld beyond 2^24", (long long)K);
    if ((double)M * N >= kMaxElements || (double)M * K >= kMaxElements || (double)N * K >= kMaxElements) return report(PDA_ERR_UNSUPPORTED, "a matrix beyond 2^40 elements");
    return PDA_OK;
}

// ---- rotary positions
int check_rope(const pda_rope* r, int d) {
    if (!r) return report(PDA_ERR_INVALID_ARG, "null rope");
    if (r->rot < 0 || r->rot > d || r->rot % 8 != 0) return report(PDA_ERR_INVALID_ARG, "rot=%d (need a multiple of 8 from 0 to d=%d)", r->rot, d);
    if (r->rot == 0) return PDA_OK;
    if (r->layout != PDA_ROPE_INTERLEAVED && r->layout != PDA_ROPE_HALF) return report(PDA_ERR_INVALID_ARG, "unknown layout=%d", r->layout);
    if (r->axes < 1 || r->axes > PDA_ROPE_MAX_AXES) return report(PDA_ERR_INVALID_ARG, "axes=%d (need 1 to %d)", r->axes, PDA_ROPE_MAX_AXES);
    int64_t sum = 0;
    for (int i = 0; i < r->axes; ++i) {
        if (r->axis_pairs[i] < 0) return report(PDA_ERR_INVALID_ARG, "axis_pairs[%d]=%d is negative", i, r->axis_pairs[i]);
        sum += r->axis_pairs[i];
    }
    if (sum != r->rot / 2) return report(PDA_ERR_INVALID_ARG, "axis_pairs sum to %lld, rot/2 is %d", (long long)sum, r->rot / 2);
    if (!r->freqs) return report(PDA_ERR_INVALID_ARG, "null freqs");
    for (int i = 0; i < r->rot / 2; ++i)
        if (!std::isfinite(r->freqs[i])) return report(PDA_ERR_INVALID_ARG, "freqs[%d] is not finite", i);
    if (r->positions) {
        if (!aligned(r->positions, 4)) return report(PDA_ERR_UNSUPPORTED, "positions must be 4-byte aligned");
        if (r->pos_batch < 0 || r->pos_batch >= (int64_t)1 << 40) return report(PDA_ERR_INVALID_ARG, "pos_batch=%lld outside [0, 2^40)", (long long)r->pos_batch);
    } else {
        if (r->axes != 1) return report(PDA_ERR_INVALID_ARG, "null positions with %d axes", r->axes);
        if (r->first < 0 || r->first >= (int64_t)1 << 40) return report(PDA_ERR_INVALID_ARG, "first=%lld outside [0, 2^40)", (long long)r->first);
    }
    return PDA_OK;
}

struct Tokens {              // a token-major tensor
    const void* p;
    int type;
    int64_t batch, token;
    const char* name;
};
int check_tokens(const Tokens& t, int B, int64_t S, int64_t n, bool written) {
    const int vec = t.type == PDA_BF16 ? 8 : 4;
    if (t.batch < 0 || t.token < 0 || t.batch >= (int64_t)1 << 40 || t.token >= (int64_t)1 << 40)
        return report(PDA_ERR_INVALID_ARG, "a stride of %s outside [0, 2^40)", t.name);
    if (t.batch % vec != 0 || t.token % vec != 0) return report(PDA_ERR_UNSUPPORTED, "strides of %s must be multiples of %d elements", t.name, vec);
    if ((double)(B - 1) * t.batch + (double)(S - 1) * t.token + n >= 4 * kMaxElements) return report(PDA_ERR_UNSUPPORTED, "%s spans more than 2^42 elements", t.name);
    if (!aligned(t.p, 16)) return report(PDA_ERR_UNSUPPORTED, "%s must be 16-byte aligned", t.name);
    if (written && S > 1 && t.token < n) return report(PDA_ERR_INVALID_ARG, "tokens of %s overlap", t.name);
    return written ? check_blocks(B, S, t.batch, t.token, n, t.name) : (int)PDA_OK;
}

int rope(const Tokens& x, const Tokens& dx, void* y, int64_t y_batch, int64_t y_head, int B, int64_t S, int H, int d,
         const pda_rope* r, int unit_rms, float premul, bool backward, void* stream) {
    const char* yn = backward ? "dy" : "y";
    if (B < 0 || H < 0 || S < 0) return report(PDA_ERR_INVALID_ARG, "negative size (B=%d H=%d S=%lld)", B, H, (long long)S);
    if (d != 64 && d != 128) return report(PDA_ERR_UNSUPPORTED, "head dim d=%d not supported (64 or 128)", d);
    if (bad_type(x.type)) return report(PDA_ERR_INVALID_ARG, "unknown x_type=%d", x.type);
    int rc = check_rope(r, d);
    if (rc != PDA_OK) return rc;
    if (!std::isfinite(premul)) return report(PDA_ERR_INVALID_ARG, "premul must be finite");
    if ((double)B * H * (double)S * d >= kMaxElements || S >= kMaxRows) return report(PDA_ERR_UNSUPPORTED, "B*H*S*d overflows 2^40 elements, or S 2^31");
    if (H >= 1 << 24) return report(PDA_ERR_UNSUPPORTED, "H=%d heads (fewer than 2^24 supported)", H);
    if (B == 0 || H == 0 || S == 0) return PDA_OK;
    const int64_t n = (int64_t)H * d, head = S * d;
    const bool reads_x = !backward || unit_rms;
    if (!y || (reads_x && !x.p) || (backward && !dx.p)) return report(PDA_ERR_INVALID_ARG, "null %s", backward ? "dy/dx, or x with unit_rms" : "x/y");
    if (y_batch < 0 || y_head < 0 || y_batch >= (int64_t)1 << 40 || y_head >= (int64_t)1 << 40) return report(PDA_ERR_INVALID_ARG, "a stride of %s outside [0, 2^40)", yn);
    if (y_batch % 8 != 0 || y_head % 8 != 0) return report(PDA_ERR_UNSUPPORTED, "strides of %s must be multiples of 8 elements", yn);
    if ((double)(B - 1) * y_batch + (double)(H - 1) * y_head + head >= 4 * kMaxElements) return report(PDA_ERR_UNSUPPORTED, "%s spans more than 2^42 elements", yn);
    if (!aligned(y, 16)) return report(PDA_ERR_UNSUPPORTED, "%s must be 16-byte aligned", yn);
    if (reads_x && (rc = check_tokens(x, B, S, n, false)) != PDA_OK) return rc;
    if (backward && (rc = check_tokens(dx, B, S, n, true)) != PDA_OK) return rc;
    if (!backward && (rc = check_blocks(B, H, y_batch, y_head, head, yn)) != PDA_OK) return rc;
    const View vy = view(y, head, 2, B, H, y_batch, y_head, yn);
    const View vx = reads_x ? view(x.p, n, type_size(x.type), B, S, x.batch, x.token, "x") : View{};
    const View vp = r->rot > 0 && r->positions ? view(r->positions, S * r->axes, 4, B, 1, r->pos_batch, 0, "positions") : View{};
    if (backward) {
        const View vd = view(dx.p, n, type_size(dx.type), B, S, dx.batch, dx.token, "dx");
        if ((rc = check_apart({vd}, {vy, vp})) != PDA_OK) return rc;
        const bool itself = dx.p == x.p && dx.batch == x.batch && dx.token == x.token;
        if (!itself && (rc = check_apart({vd}, {vx})) != PDA_OK) return rc;
    } else if ((rc = check_apart({vy}, {vx, vp})) != PDA_OK) {
        return rc;
    }
    RopeParams p{};
    p.x = x.p; p.dx = const_cast<void*>(dx.p); p.y = static_cast<__bf16*>(y);
    p.x_batch = x.batch; p.x_token = x.token; p.dx_batch = dx.batch; p.dx_token = dx.token;
    p.y_batch = y_batch; p.y_head = y_head;
    p.S = S; p.B = B; p.H = H;
    p.x_bf16 = x.type == PDA_BF16; p.unit_rms = unit_rms != 0; p.premul = premul;
    p.rot = r->rot;
    if (r->rot > 0) {
        p.layout = r->layout; p.axes = r->axes;
        p.positions = r->positions; p.pos_batch = r->pos_batch; p.first = r->first;
        for (int i = 0, sum = 0; i < r->axes; ++i) p.axis_end[i] = sum += r->axis_pairs[i];
        for (int i = 0; i < r->rot / 2; ++i) p.turns[i] = r->freqs[i] / 6.283185307179586476925;
    }
    int n_cu = 0;
    hipError_t e = device_cu_count(&n_cu);
    if (e != hipSuccess) return hip_error(e, "device query");
    e = launch_rope(p, d, backward, n_cu, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)PDA_OK : hip_error(e, backward ? "rotary pack gradient launch" : "rotary pack launch");
}

}  // namespace

extern "C" {

int pda_fp8_quant(const void* x, int x_type, int64_t rows, int64_t cols, int64_t ldx, int fp8_type, int block_rows,
                  void* q, uint8_t* q_scales, void* qt, uint8_t* qt_scales, void* stream) {
    if (bad_type(x_type)) return report(PDA_ERR_INVALID_ARG, "unknown x_type=%d", x_type);
    if (bad_fp8(fp8_type)) return report(PDA_ERR_INVALID_ARG, "unknown fp8_type=%d", fp8_type);
    if (block_rows != 1 && block_rows != 128) return report(PDA_ERR_INVALID_ARG, "block_rows=%d (need 1 or 128)", block_rows);
    if (rows < 0 || cols < 0 || ldx < cols) return report(PDA_ERR_INVALID_ARG, "rows=%lld cols=%lld ldx=%lld (need >= 0, ldx >= cols)", (long long)rows, (long long)cols, (long long)ldx);
    if (rows >= kMaxRows || cols >= kMaxRows || (double)rows * ldx >= kMaxElements || (double)(rows + 128) * (cols + 128) >= kMaxElements)
        return report(PDA_ERR_UNSUPPORTED, "rows or cols beyond 2^31, or a matrix beyond 2^40 elements");
    if (!q != !q_scales || !qt != !qt_scales) return report(PDA_ERR_INVALID_ARG, "values and scales go together");
    if (!q && !qt) return report(PDA_ERR_INVALID_ARG, "null q and qt: nothing to compute");
    if (rows == 0 || cols == 0) return PDA_OK;
    if (!x) return report(PDA_ERR_INVALID_ARG, "null x");
    if (!aligned(x, type_size(x_type))) return report(PDA_ERR_UNSUPPORTED, "x must be aligned to its element");
    if (!aligned(q, 16) || !aligned(qt, 16)) return report(PDA_ERR_UNSUPPORTED, "q/qt must be 16-byte aligned");
    if (!aligned(q_scales, 4) || !aligned(qt_scales, 4)) return report(PDA_ERR_UNSUPPORTED, "scales must be 4-byte aligned");
    const int64_t rb = block_rows == 1 ? rows : (rows + 127) / 128, cb = block_rows == 1 ? cols : (cols + 127) / 128;
    const Range rx{x, ((double)(rows - 1) * ldx + cols) * type_size(x_type), "x"}, rq{q, (double)rows * fp8_cols(cols), "q"},
        rqs{q_scales, (double)rb * fp8_scale_cols(cols), "q_scales"}, rt{qt, (double)cols * fp8_cols(rows), "qt"},
        rts{qt_scales, (double)cb * fp8_scale_cols(rows), "qt_scales"};
    int rc;
    if ((rc = check_apart({rq, rqs, rt, rts}, {rx})) != PDA_OK || (rc = check_apart({rq}, {rqs, rt, rts})) != PDA_OK ||
        (rc = check_apart({rqs}, {rt, rts})) != PDA_OK || (rc = check_apart({rt}, {rts})) != PDA_OK) return rc;
    QuantParams p{};
    p.x = x; p.q = q; p.q_scales = q_scales; p.qt = qt; p.qt_scales = qt_scales;
    p.rows = rows; p.cols = cols; p.ldx = ldx;
    p.x_bf16 = x_type == PDA_BF16; p.e5m2 = fp8_type == PDA_E5M2; p.square = block_rows == 128;
    const hipError_t e = launch_fp8_quant(p, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)PDA_OK : hip_error(e, "quantisation launch");
}

int pda_fp8_matmul_workspace(int64_t M, int64_t N, int64_t K, int n_cu, int64_t* bytes) {
    const int rc = check_matmul(M, N, K);
    if (rc != PDA_OK) return rc;
    if (n_cu < 0) return report(PDA_ERR_INVALID_ARG, "n_cu=%d is negative", n_cu);
    if (!bytes) return report(PDA_ERR_INVALID_ARG, "null bytes");
    if (n_cu == 0) {
        const hipError_t e = device_cu_count(&n_cu);
        if (e != hipSuccess) return hip_error(e, "device query");
    }
    *bytes = M == 0 || N == 0 || K == 0 ? 0 : matmul_workspace_bytes(plan_matmul(M, N, K, n_cu), M, N);
    return PDA_OK;
}

int pda_fp8_matmul(const void* a, int a_type, const uint8_t* a_scales, const void* b, const uint8_t* b_scales, int b_block_rows,
                   const float* bias, void* out, int64_t M, int64_t N, int64_t K, int64_t ldo,
                   void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_matmul(M, N, K);
    if (rc != PDA_OK) return rc;
    if (bad_fp8(a_type)) return report(PDA_ERR_INVALID_ARG, "unknown a_type=%d", a_type);
    if (b_block_rows != 1 && b_block_rows != 128) return report(PDA_ERR_INVALID_ARG, "b_block_rows=%d (need 1 or 128)", b_block_rows);
    if (ldo < N || ldo >= (int64_t)1 << 40 || (double)M * ldo >= kMaxElements) return report(PDA_ERR_INVALID_ARG, "ldo=%lld (need >= N, M*ldo below 2^40)", (long long)ldo);
    if (M == 0 || N == 0) return PDA_OK;
    if (!out || (K > 0 && (!a || !b || !a_scales || !b_scales))) return report(PDA_ERR_INVALID_ARG, "null a/b/scales/out");
    if (!aligned(a, 16) || !aligned(b, 16) || !aligned(out, 16)) return report(PDA_ERR_UNSUPPORTED, "a/b/out must be 16-byte aligned");
    if (!aligned(a_scales, 4) || !aligned(b_scales, 4) || !aligned(bias, 4)) return report(PDA_ERR_UNSUPPORTED, "scales and bias must be 4-byte aligned");
    const int64_t sc = fp8_scale_cols(K), nb = b_block_rows == 1 ? N : (N + 127) / 128;
    const Range ro{out, ((double)(M - 1) * ldo + N) * 2, "out"};
    const std::initializer_list<Range> in = {{K ? a : nullptr, (double)M * K, "a"}, {K ? b : nullptr, (double)N * K, "b"}, {K ? a_scales : nullptr, (double)M * sc, "a_scales"},
                                             {K ? b_scales : nullptr, (double)nb * sc, "b_scales"}, {bias, (double)N * 4, "bias"}};
    if ((rc = check_apart({ro}, in)) != PDA_OK) return rc;
    MatmulParams p{};
    p.a = static_cast<const unsigned char*>(a);
    p.b = static_cast<const unsigned char*>(b);
    p.a_scales = a_scales; p.b_scales = b_scales; p.bias = bias;
    p.out = static_cast<__bf16*>(out);
    p.M = M; p.N = N; p.K = K; p.ldo = ldo;
    p.scale_cols = sc;
    p.b_shift = b_block_rows == 128 ? 7 : 0;
    p.e5m2 = a_type == PDA_E5M2;
    int n_cu = 0;
    hipError_t e = device_cu_count(&n_cu);
    if (e != hipSuccess) return hip_error(e, "device query");
    const MatmulPlan w = plan_matmul(M, N, K, n_cu);
    const int64_t need = K > 0 ? matmul_workspace_bytes(w, M, N) : 0;
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return report(PDA_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed", workspace ? (long long)workspace_bytes : 0LL, (long long)need);
        if (!aligned(workspace, 256)) return report(PDA_ERR_UNSUPPORTED, "workspace must be 256-byte aligned");
        const Range ws{workspace, (double)need, "workspace"};
        if ((rc = check_apart({ws}, in)) != PDA_OK || (rc = check_apart({ws}, {ro})) != PDA_OK) return rc;
        p.part = static_cast<float*>(workspace);
    }
    e = launch_fp8_matmul(p, w, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)PDA_OK : hip_error(e, "8-bit product launch");
}

int pda_rms_norm_fwd(const void* x, int x_type, const void* res, int res_type, const float* weight, void* h, void* y, int y_type,
                     uint8_t* y_scales, float* rstd, int64_t rows, int64_t groups, int D, float eps, void* stream) {
    int rc = check_rms(rows, groups, D);
    if (rc != PDA_OK) return rc;
    if (bad_type(x_type) || (res && bad_type(res_type)) || (bad_type(y_type) && y_type != PDA_E4M3))
        return report(PDA_ERR_INVALID_ARG, "unknown type (x_type=%d res_type=%d y_type=%d)", x_type, res_type, y_type);
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return report(PDA_ERR_INVALID_ARG, "eps must be finite and >= 0");
    const bool fp8 = y_type == PDA_E4M3;
    if (rows == 0) return PDA_OK;
    if (!res != !h) return report(PDA_ERR_INVALID_ARG, "res and h go together");
    if (fp8 != (y_scales != nullptr)) return report(PDA_ERR_INVALID_ARG, "y_scales go with an 8-bit y");
    if (!x || !y) return report(PDA_ERR_INVALID_ARG, "null x/y");
    if (!aligned(x, 16) || !aligned(res, 16) || !aligned(h, 16) || !aligned(y, 16) || !aligned(weight, 16)) return report(PDA_ERR_UNSUPPORTED, "x/res/h/y/weight must be 16-byte aligned");
    if (!aligned(y_scales, 4) || !aligned(rstd, 4)) return report(PDA_ERR_UNSUPPORTED, "y_scales/rstd must be 4-byte aligned");
    const double n = (double)rows * D;
    const Range rx{x, n * type_size(x_type), "x"}, rr{res, res ? n * type_size(res_type) : 0, "res"}, rh{h, rr.bytes, "h"},
        ry{y, fp8 ? (double)rows * fp8_cols(D) : n * type_size(y_type), "y"}, rs{y_scales, fp8 ? (double)rows * fp8_scale_cols(D) : 0, "y_scales"},
        rd{rstd, (double)rows * 4, "rstd"}, rw{weight, (double)groups * D * 4, "weight"};
    if ((rc = check_itself(rh, res_type, rx, x_type)) != PDA_OK || (rc = check_itself(rh, res_type, rr, res_type)) != PDA_OK) return rc;
    if ((rc = check_apart({rh}, {rw})) != PDA_OK || (rc = check_apart({ry, rs, rd}, {rx, rr, rw, rh})) != PDA_OK ||
        (rc = check_apart({ry}, {rs, rd})) != PDA_OK || (rc = check_apart({rs}, {rd})) != PDA_OK) return rc;
    RmsNormParams p{};
    p.x = x; p.res = res; p.weight = weight; p.h = h; p.y = y; p.y_scales = y_scales; p.rstd = rstd;
    p.rows = rows; p.groups = groups; p.group_rows = rows / groups; p.D = D; p.eps = eps;
    p.x_type = x_type; p.h_type = res_type; p.y_type = y_type;
    const hipError_t e = launch_rms_norm_fwd(p, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)PDA_OK : hip_error(e, "rms norm launch");
}

int pda_rms_norm_bwd_workspace(int64_t rows, int64_t groups, int D, int n_cu, int64_t* bytes) {
    const int rc = check_rms(rows, groups, D);
    if (rc != PDA_OK) return rc;
    if (n_cu < 0) return report(PDA_ERR_INVALID_ARG, "n_cu=%d is negative", n_cu);
    if (!bytes) return report(PDA_ERR_INVALID_ARG, "null bytes");
    if (n_cu == 0) {
        const hipError_t e = device_cu_count(&n_cu);
        if (e != hipSuccess) return hip_error(e, "device query");
    }
    *bytes = rms_workspace_bytes(rows, groups, D, n_cu);
    return PDA_OK;
}

int pda_rms_norm_bwd(const void* dy, int dy_type, const void* h, int h_type, const float* weight, const float* rstd, const void* dres,
                     void* dh, float* dweight, int64_t rows, int64_t groups, int D, void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_rms(rows, groups, D);
    if (rc != PDA_OK) return rc;
    if (bad_type(dy_type) || bad_type(h_type)) return report(PDA_ERR_INVALID_ARG, "unknown type (dy_type=%d h_type=%d)", dy_type, h_type);
    if (!dh && !dweight) return report(PDA_ERR_INVALID_ARG, "null dh and dweight: nothing to compute");
    if (!aligned(weight, 16) || !aligned(dweight, 16)) return report(PDA_ERR_UNSUPPORTED, "weight/dweight must be 16-byte aligned");
    if (rows == 0 && !dweight) return PDA_OK;
    RmsNormParams p{};
    if (rows > 0) {
        if (!dy || !h || !rstd) return report(PDA_ERR_INVALID_ARG, "null dy/h/rstd");
        if (!aligned(dy, 16) || !aligned(h, 16) || !aligned(dres, 16) || !aligned(dh, 16)) return report(PDA_ERR_UNSUPPORTED, "dy/h/dres/dh must be 16-byte aligned");
        if (!aligned(rstd, 4)) return report(PDA_ERR_UNSUPPORTED, "rstd must be 4-byte aligned");
        const double n = (double)rows * D, param = (double)groups * D * 4;
        const Range ry{dy, n * type_size(dy_type), "dy"}, rh{h, n * type_size(h_type), "h"}, rr{dres, rh.bytes, "dres"}, rd{dh, rh.bytes, "dh"},
            rw{dweight, param, "dweight"}, in_w{weight, param, "weight"}, in_s{rstd, (double)rows * 4, "rstd"};
        if ((rc = check_itself(rd, h_type, ry, dy_type)) != PDA_OK || (rc = check_itself(rd, h_type, rh, h_type)) != PDA_OK || (rc = check_itself(rd, h_type, rr, h_type)) != PDA_OK) return rc;
        if ((rc = check_apart({rd, rw}, {in_w, in_s})) != PDA_OK || (rc = check_apart({rw}, {ry, rh, rr, rd})) != PDA_OK) return rc;
        int n_cu = 0;
        const hipError_t e = device_cu_count(&n_cu);
        if (e != hipSuccess) return hip_error(e, "device query");
        const int64_t need = dweight ? rms_workspace_bytes(rows, groups, D, n_cu) : 0;
        if (need > 0 && (!workspace || workspace_bytes < need))
            return report(PDA_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed", workspace ? (long long)workspace_bytes : 0LL, (long long)need);
        if (need > 0 && !aligned(workspace, 16)) return report(PDA_ERR_UNSUPPORTED, "workspace must be 16-byte aligned");
        const Range ws{need > 0 ? workspace : nullptr, (double)need, "workspace"};
        if ((rc = check_apart({ws}, {ry, rh, rr, rd, rw, in_w, in_s})) != PDA_OK) return rc;
        p.group_rows = rows / groups;
        p.chunks = ln_chunks(p.group_rows, groups, D, n_cu);
    }
    p.x = dy; p.h = const_cast<void*>(h); p.res = dres; p.weight = weight; p.y = dh; p.rstd = const_cast<float*>(rstd);
    p.dweight = dweight; p.part = static_cast<float*>(workspace);
    p.rows = rows; p.groups = groups; p.D = D;
    p.x_type = dy_type; p.h_type = h_type;
    const hipError_t e = launch_rms_norm_bwd(p, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? (int)PDA_OK : hip_error(e, "rms norm gradient launch");
}

int pda_pack_heads_rope(const void* x, int x_type, int64_t x_batch, int64_t x_token, void* y, int64_t y_batch, int64_t y_head,
                        int B, int64_t S, int H, int d, const pda_rope* r, int unit_rms, float premul, void* stream) {
    return rope({x, x_type, x_batch, x_token, "x"}, {nullptr, x_type, 0, 0, "dx"}, y, y_batch, y_head, B, S, H, d, r, unit_rms, premul, false, stream);
}

int pda_pack_heads_rope_bwd(const void* dy, int64_t dy_batch, int64_t dy_head, const void* x, int x_type, int64_t x_batch, int64_t x_token,
                            void* dx, int64_t dx_batch, int64_t dx_token, int B, int64_t S, int H, int d,
                            const pda_rope* r, int unit_rms, float premul, void* stream) {
    return rope({x, x_type, x_batch, x_token, "x"}, {dx, x_type, dx_batch, dx_token, "dx"}, const_cast<void*>(dy), dy_batch, dy_head, B, S, H, d, r, unit_rms, premul, true, stream);
}

int pda_rope_frequencies(int n, double base, int scaling, double factor, double original, double slow_turns, double fast_turns,
                         double* freqs, double* magnitude) {
    if (n < 1 || n > 1 << 20) return report(PDA_ERR_INVALID_ARG, "n=%d pairs (need 1 to 2^20)", n);
    if (!(base > 1.0) || !std::isfinite(base)) return report(PDA_ERR_INVALID_ARG, "base must be finite and > 1");
    if (scaling < PDA_ROPE_PLAIN || scaling > PDA_ROPE_BLEND) return report(PDA_ERR_INVALID_ARG, "unknown scaling=%d", scaling);
    if (!freqs) return report(PDA_ERR_INVALID_ARG, "null freqs");
    if (scaling != PDA_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return report(PDA_ERR_INVALID_ARG, "factor must be finite and >= 1");
    if (scaling == PDA_ROPE_BLEND && (!(original > 0.0) || !std::isfinite(original) || !(slow_turns >= 0.0) || !(fast_turns > slow_turns) || !std::isfinite(fast_turns)))
        return report(PDA_ERR_INVALID_ARG, "need original > 0 and 0 <= slow_turns < fast_turns, all finite");
    const double b = scaling == PDA_ROPE_BASE && n > 1 ? base * std::pow(factor, (double)n / (n - 1)) : base;
    for (int i = 0; i < n; ++i) {
        double f = std::pow(b, -(double)i / n);
        if (scaling == PDA_ROPE_LINEAR) f /= factor;
        if (scaling == PDA_ROPE_BLEND) {
            const double share = (original * f / 6.283185307179586476925 - slow_turns) / (fast_turns - slow_turns);
            const double keep = share < 0.0 ? 0.0 : share > 1.0 ? 1.0 : share;
            f = f * keep + f / factor * (1.0 - keep);
        }
        freqs[i] = f;
    }
    if (magnitude) *magnitude = scaling == PDA_ROPE_BLEND ? 0.1 * std::log(factor) + 1.0 : 1.0;
    return PDA_OK;
}

}  // extern "C"
