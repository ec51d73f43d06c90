// Internal declarations of the training operators (not part of the ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pda {

// Sets the calling thread's error message and returns `code` (api.hip).
int report(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// ---- attention, backward (attn_bwd.hip) ---------------------------------------------------------
constexpr int kBwdTile = 32;            // streamed rows of a step
constexpr int kBwdRows = 256;           // resident rows of a workgroup

// The work items of a launch, in the order in which they start: the blocks of 256 valid keys (dk and dv; a step is four products), each
// against `key_parts` ranges of the query rows; the blocks of 256 query rows (dq; three products), the last `query_cut` of them each
// against `query_parts` ranges of the keys; blocks of hidden keys only (zeros).
struct BwdPlan {
    int key_per_head, query_per_head;   // blocks
    int key_blocks, query_blocks;       // of all heads
    int key_parts;                      // 1: none is cut
    int query_cut, query_parts;         // 0, 1: none is cut
};
constexpr int kBwdMaxParts = 16;
// Steps of a block against n streamed rows.
inline int64_t bwd_steps(int64_t n) { return (n + kBwdTile - 1) / kBwdTile; }
// Time of an item in tenths of a query step (1.3 us at d = 128, 0.8 at 64): a key step takes 1.2 of it, start and end of an item about six.
inline int64_t bwd_key_time(int64_t steps) { return steps * 12 + 60; }
inline int64_t bwd_query_time(int64_t steps) { return steps * 10 + 60; }
// Partial sums of kBwdRows rows and d columns that a plan writes and a second kernel adds: written and read at about 4 TB/s, and that
// kernel's launch.
inline int64_t bwd_part_slots(const BwdPlan& w) { return (w.key_parts > 1 ? (int64_t)w.key_blocks * w.key_parts * 2 : 0) + (int64_t)w.query_cut * (w.query_cut ? w.query_parts : 0); }
inline int64_t bwd_join_time(const BwdPlan& w, int d) { const int64_t n = bwd_part_slots(w); return n ? 30 + n * d / 200 : 0; }
// When the last item of a launch ends if each goes, in order, to the compute unit that is free first.
inline int64_t bwd_end(const BwdPlan& w, int64_t Sq, int64_t n_v, int n_cu) {
    struct Free { int64_t at, units; } f[8] = {{0, n_cu}};     // compute units by the time at which they become free
    int groups = 1;
    const int64_t sk = bwd_steps(Sq), sq = bwd_steps(n_v);
    const struct { int64_t n, time; } jobs[3] = {{(int64_t)w.key_blocks * w.key_parts, bwd_key_time((sk + w.key_parts - 1) / w.key_parts)},
                                                 {w.query_blocks - w.query_cut, bwd_query_time(sq)},
                                                 {(int64_t)w.query_cut * w.query_parts, bwd_query_time((sq + w.query_parts - 1) / w.query_parts)}};
    int64_t end = 0;
    for (const auto& j : jobs) {
        for (int64_t left = j.n; left > 0;) {
            int g = 0, last = 0;
            for (int i = 1; i < groups; ++i) {
                g = f[i].at < f[g].at ? i : g;
                last = f[i].at > f[last].at ? i : last;
            }
            if (left >= n_cu && f[last].at - f[g].at <= j.time) {      // whole rounds: each unit takes one item, and all are as far apart as before
                const int64_t rounds = left / n_cu;
                for (int i = 0; i < groups; ++i) f[i].at += rounds * j.time;
                if (f[last].at > end) end = f[last].at;
                left -= rounds * n_cu;
                continue;
            }
            const int64_t n = f[g].units < left ? f[g].units : left;
            int64_t rounds = 1;                                // of the first group alone, up to the next one's time
            if (n == f[g].units) {
                int64_t next = f[last].at;
                for (int i = 0; i < groups; ++i)
                    if (i != g && f[i].at < next) next = f[i].at;
                const int64_t reach = (next - f[g].at + j.time - 1) / j.time, most = left / n;
                if (reach > 1) rounds = reach < most ? reach : most;
            }
            const int64_t at = f[g].at + rounds * j.time;
            left -= n * rounds;
            if (at > end) end = at;
            int same = 0;
            while (same < groups && f[same].at != at) ++same;
            if (n == f[g].units && same == groups) f[g].at = at;               // all of them
            else {
                f[g].units -= n;
                if (same < groups) f[same].units += n;
                else f[groups++] = {at, n};
                if (f[g].units == 0) f[g] = f[--groups];
            }
        }
    }
    return end;
}
// Cuts.  A launch of fewer blocks than compute units is cut so that its parts fill them in one round, key and query blocks into parts of
// about equal time; one of more blocks has the blocks that start last cut where that ends it earlier, and its key blocks, which start
// first, where there are few of them against many rows.  Candidates are compared by bwd_end and the time of the second kernel: 0.1 to
// 4 us of host time in all, up to 16 where there are many query blocks against few keys.
// us, uncut -> cut: d = 128: 1 x 9 600 343 -> 157, 12 x 3 000 240 -> 191, 24 x 2 048 184 -> 172, 24 x 16 384 on 570 628 -> 461, 24 x 9 600 3 329 -> 3 131,
// 3 x 67 576 20 132 -> 18 822; d = 64: 2 x 1 024 39 -> 22, 1 x 9 600 294 -> 113, 24 x 4 797 569 -> 545, 6 x 33 000 6 891 -> 6 020 (all but
// 12 x 3 000 before workgroups took their items from a counter).
inline BwdPlan plan_bwd(int64_t Sq, int64_t n_v, int64_t BH, int d, int n_cu) {
    BwdPlan w{};
    w.key_per_head = (int)((n_v + kBwdRows - 1) / kBwdRows);
    w.query_per_head = (int)((Sq + kBwdRows - 1) / kBwdRows);
    w.key_blocks = (int)(BH * w.key_per_head);
    w.query_blocks = (int)(BH * w.query_per_head);
    w.key_parts = w.query_parts = 1;
    const int64_t sk = bwd_steps(Sq), sq = bwd_steps(n_v), blocks = (int64_t)w.key_blocks + w.query_blocks;
    if (w.key_blocks == 0 || w.query_blocks == 0) return w;
    const int64_t key_time = bwd_key_time(sk), query_time = bwd_query_time(sq), longest = key_time > query_time ? key_time : query_time;
    // so long a launch has nothing to gain at its end, unless that is a few blocks against the long side among many against the short one
    if (blocks > 64 * (int64_t)n_cu && longest * 16 * n_cu <= w.key_blocks * key_time + w.query_blocks * query_time) return w;
    // two steps a part at the least; one part is always a candidate, so that query blocks are cut where key blocks cannot be
    const int max_k = (int)(sk < 4 ? 1 : sk / 2 < kBwdMaxParts ? sk / 2 : kBwdMaxParts), max_q = (int)(sq / 2 < kBwdMaxParts ? sq / 2 : kBwdMaxParts);
    BwdPlan best = w;
    int64_t best_time = bwd_end(w, Sq, n_v, n_cu);
    // One tile of query rows and few keys: over before the host has issued another kernel (17 rows, one head, uncut and cut, us: d = 64 on 256 keys 13.7 and 16.3,
    // 384 14.9 and 16.3, 448 16.2 and 16.3, 640 20.0 and 16.3; d = 128 on 256 keys 16.6 and 16.2, 640 28.1 and 17.4).
    if (sk == 1 && best_time <= (d == 64 ? 190 : 120)) return w;
    auto consider = [&](int key_parts, int query_cut, int query_parts) {
        BwdPlan c = w;
        c.key_parts = key_parts;
        if (query_parts > 1) {
            c.query_cut = query_cut;
            c.query_parts = query_parts;
        }
        if (bwd_part_slots(c) > 4 * (int64_t)n_cu) return;
        const int64_t t = bwd_end(c, Sq, n_v, n_cu) + bwd_join_time(c, d);
        if (t < best_time) {
            best = c;
            best_time = t;
        }
    };
    if (blocks <= n_cu) {
        for (int k = 1; k <= max_k && w.key_blocks * k + w.query_blocks <= n_cu; ++k) {
            const int64_t most = (n_cu - (int64_t)w.key_blocks * k) / w.query_blocks, even = (sq * 10 * k + sk * 12 - 1) / (sk * 12);
            const int64_t q = most < max_q ? most : max_q;
            consider(k, w.query_blocks, (int)q);
            if (q > 1) {
                const int64_t steps = (sq + q - 1) / q, least = (sq + steps - 1) / steps;      // the fewest parts that are as short
                if (least < q) consider(k, w.query_blocks, (int)least);
            }
            if (even < q) consider(k, w.query_blocks, (int)even);
            if (even - 1 < q) consider(k, w.query_blocks, (int)(even - 1));
        }
        return best;
    }
    for (int k = 1; k <= max_k && (k == 1 || (int64_t)w.key_blocks * k <= 2 * (int64_t)n_cu); ++k) {
        if (k > 1) consider(k, 0, 1);
        for (int r = k == 1 ? 1 : 4; r <= 16; r += r < 4 ? 1 : 4) {        // sixteenths of the compute units
            const int64_t cut = r * (int64_t)n_cu / 16;
            if (cut == 0) continue;
            const bool all = cut >= w.query_blocks;            // few query blocks: each part of them counts
            for (int q = 2; q <= (all ? kBwdMaxParts : k == 1 && r <= 4 ? 8 : 4) && q <= max_q; ++q) consider(k, all ? w.query_blocks : (int)cut, q);
            if (all) break;
        }
    }
    return best;
}
__host__ __device__ inline int64_t bwd_key_floats(const BwdPlan& w, int d) { return w.key_parts > 1 ? (int64_t)w.key_blocks * w.key_parts * 2 * kBwdRows * d : 0; }

struct AttnBwdParams {
    const __bf16* dout;
    const __bf16* q;
    const __bf16* k;
    const __bf16* v;
    const void* out;
    const float* lse;
    __bf16* dq;
    __bf16* dk;
    __bf16* dv;
    float* stats;            // d = 128: [B*H][stat_rows / 32][2][32]: -lse * log2(e) of 32 rows (-inf where a row has no keys and behind the last row),
                             // -<dout, out> of the same rows (0 there).  d = 64: [B*H][stat_rows][8] bf16, three whose sum is -lse / scale (-2^100 there)
                             // and a zero, three whose sum is -<dout, out> and a zero
    int64_t Sq, Skv, n_v;    // query rows, key rows, valid keys
    int64_t stat_rows;       // bwd_stat_rows(Sq)
    int64_t do_bs, do_hs, q_bs, q_hs, kv_bs, kv_hs, o_bs, o_hs, l_bs, l_hs, dq_bs, dq_hs, dkv_bs, dkv_hs;
    int B, H;
    int out_bf16;
    float scale, scale_log2e;
    float* parts;            // partial sums of cut blocks: the key blocks' (dk, dv of a part, part after part, block after block), the query blocks'
    BwdPlan plan;
    int* counter;            // items taken beyond each workgroup's first; set to zero by the statistics' kernel
    int items, grid, n_cu;   // work items, workgroups, compute units
};
inline int64_t bwd_stat_rows(int64_t Sq) { return (Sq + 63) / 64 * 64; }
// The counter, then the statistics.
constexpr int64_t kBwdCounterBytes = 256;
inline int64_t bwd_stat_bytes(int64_t BH, int64_t Sq, int d) { return Sq == 0 ? 0 : kBwdCounterBytes + (BH * bwd_stat_rows(Sq) * (d == 64 ? 16 : 8) + 255) / 256 * 256; }
inline int64_t bwd_workspace_bytes(const BwdPlan& w, int64_t BH, int64_t Sq, int d) { return bwd_stat_bytes(BH, Sq, d) + bwd_part_slots(w) * kBwdRows * d * 4; }
// Enough for every plan of at most these sizes: a plan has kBwdMaxParts parts a block and two steps a part at the least, 4 n_cu slots at the most.
inline int64_t bwd_workspace_bound(int64_t BH, int64_t Sq, int64_t Skv, int d, int n_cu) {
    const auto parts = [](int64_t n) { const int64_t p = bwd_steps(n) / 2; return p < 2 ? 0 : p < kBwdMaxParts ? p : kBwdMaxParts; };
    const auto blocks = [BH](int64_t n) { return BH * ((n + kBwdRows - 1) / kBwdRows); };
    const int64_t slots = blocks(Skv) * parts(Sq) * 2 + blocks(Sq) * parts(Skv), most = 4 * (int64_t)n_cu;
    return bwd_stat_bytes(BH, Sq, d) + (slots < most ? slots : most) * kBwdRows * d * 4;
}
hipError_t launch_attn_bwd(AttnBwdParams p, int d, hipStream_t st);

// ---- layer norm (layer_norm.hip) ----------------------------------------------------------------
struct LayerNormParams {
    const void* x;
    const void* dy;          // backward
    const float* weight;     // nullable
    const float* bias;       // nullable, forward
    void* y;                 // forward: y; backward: dx (nullable)
    float* mean;
    float* rstd;
    float* dweight;          // nullable
    float* dbias;            // nullable
    float* part;             // [groups][chunks][2][D] partial sums of dweight and dbias
    int64_t rows, group_rows;
    int64_t groups;
    int64_t chunks;          // backward: workgroups of a group
    int D;
    float eps;
};
hipError_t launch_layer_norm_fwd(const LayerNormParams& p, bool x_bf16, bool y_bf16, hipStream_t st);
hipError_t launch_layer_norm_bwd(const LayerNormParams& p, bool x_bf16, bool y_bf16, hipStream_t st);

// Workgroups of a group of rows in the backward kernel: as many as a compute unit holds at once (by their registers; more would leave
// the last round partly empty: 119 056 x 1 536 on 1 024 workgroups 334 us, on 1 280 346, on 2 048 380; 100 000 x 1 024 on 1 024 163, on 2 048 131;
// 4 797 x 4 096 bf16 on 1 024 33.5, on 512 26.5; 4 797 x 8 192 on 1 024 63.9, on 512 49.2, on 256 42.4), each with four rows at least, or
// up to D = 128 with the eight or 16 that it takes at once.  Where a wavefront has
// rows of its own, up to D = 512, six for each of them if all compute units then have a workgroup: 9 600 x 256 with four in all 15.2 us, with 24 10.0; 1 000 x 512
// 8.0 and 10.0.
inline int64_t ln_chunks(int64_t group_rows, int64_t groups, int D, int n_cu) {
    const int64_t per_cu = D <= 256 ? 8 : D <= 512 ? 4 : D <= 1024 ? 8 : D <= 2048 ? 4 : D <= 4096 ? 2 : 1;
    const int64_t resident = per_cu * n_cu, want = resident / groups > 1 ? resident / groups : 1;
    const int64_t least = D <= 64 ? 16 : D <= 128 ? 8 : 4;     // rows of a workgroup: what it holds at once up to D = 512
    int64_t most = (group_rows + least - 1) / least;
    if (D <= 512) {
        const int64_t each = (n_cu + groups - 1) / groups, full = (group_rows + 6 * least - 1) / (6 * least), few = each > full ? each : full;
        if (few < most) most = few;
    }
    return want < most ? want : most;
}
// One workgroup per group writes its sums itself.
inline int64_t ln_workspace_bytes(int64_t rows, int64_t groups, int D, int n_cu) {
    if (rows == 0 || groups == 0) return 0;
    const int64_t c = ln_chunks(rows / groups, groups, D, n_cu);
    return c <= 1 ? 0 : groups * c * 2 * D * 4;
}

// ---- pack, backward (layout.hip) ----------------------------------------------------------------
hipError_t launch_pack_bwd(const void* dy, const float* x, float* dx, int B, int64_t S, int H, int d, int unit_rms, float premul, hipStream_t st);

}  // namespace pda
