// C entry points of the learner operators: argument checks, workspaces and
// launch sequences.
#include "internal.hpp"

#include <cmath>
#include <cstring>

using namespace malib;

namespace {

#define HIP_TRY(expr)                                                                     \
    do {                                                                                  \
        hipError_t e_ = (expr);                                                           \
        if (e_ != hipSuccess)                                                             \
            return set_error(e_ == hipErrorOutOfMemory ? MALIB_E_NOMEM : MALIB_E_HIP,     \
                             "%s failed: %s", #expr, hipGetErrorString(e_));              \
    } while (0)

#define TRY(expr)                  \
    do {                           \
        malib_status s_ = (expr);  \
        if (s_ != MALIB_OK)        \
            return s_;             \
    } while (0)

constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 1;
constexpr int64_t kMaxWidth = (int64_t)1 << 24;
constexpr int64_t kMaxValues = (int64_t)1 << 46;   // of y or dy: sizes in bytes fit 64 bits
constexpr int64_t kFusedMost = (int64_t)1 << 20, kFusedWidth = 128;   // see BackwardPlan

int type_size(int dtype) { return dtype == MALIB_DT_BF16 ? 2 : 4; }

int64_t align256(int64_t n) { return (n + 255) / 256 * 256; }

malib_status check_linear(const malib_linear_desc* d)
{
    if (!d)
        return set_error(MALIB_E_INVAL, "desc is NULL");
    if (d->dtype != MALIB_DT_F32 && d->dtype != MALIB_DT_BF16)
        return set_error(MALIB_E_INVAL, "unknown dtype %d", d->dtype);
    if (d->act < MALIB_ACT_NONE || d->act > MALIB_ACT_SILU)
        return set_error(MALIB_E_INVAL, "unknown activation %d", d->act);
    if (d->groups < 1 || d->groups > 65535)
        return set_error(MALIB_E_INVAL, "groups must be in [1, 65535]");
    if (d->rows < 0 || d->rows > kMaxRows)
        return set_error(MALIB_E_INVAL, "rows must be in [0, 2^31)");
    if (d->in < 1 || d->in > kMaxWidth || d->out < 1 || d->out > kMaxWidth)
        return set_error(MALIB_E_INVAL, "in and out must be in [1, 2^24]");
    if (d->groups * d->rows > kMaxValues / d->out)
        return set_error(MALIB_E_UNSUPPORTED, "groups * rows * out must be at most 2^46");
    return MALIB_OK;
}

// Whether any two rows of different groups share an element (rows of one group do not)
bool groups_overlap(const malib_mat& m, int64_t rows, int64_t cols, int64_t groups)
{
    const __int128 row = rows > 1 ? m.row_stride : 0, group = m.group_stride;
    if (groups == 1 || rows == 0 || group >= (rows - 1) * row + cols)   // one behind the other
        return false;
    if (rows == 1)
        return true;
    if (group >= cols && (groups - 1) * group + cols <= row)   // side by side within a stride
        return false;
    for (int64_t g = 1; g < groups; ++g) {   // the rows of a group around row 0 of one g further
        const __int128 at = g * group, r = std::min<__int128>(at / row, rows - 1);
        if (at - r * row < cols || (r + 1 < rows && (r + 1) * row - at < cols))
            return true;
    }
    return false;
}

// A matrix argument: alignment to its element, a row stride that holds its
// columns; an output's groups must lie apart.
malib_status check_mat(const malib_mat* m, const char* what, int64_t rows, int64_t cols,
                       int64_t groups, int size, bool output)
{
    if (!m || !m->ptr)
        return set_error(MALIB_E_INVAL, "%s is NULL", what);
    if ((uintptr_t)m->ptr % size)
        return set_error(MALIB_E_INVAL, "%s is not aligned to its elements", what);
    if (rows > 1 && m->row_stride < (output ? cols : 0))
        return set_error(MALIB_E_INVAL, "%s: row stride %lld is below %lld columns", what,
                         (long long)m->row_stride, (long long)cols);
    if (m->group_stride < 0)
        return set_error(MALIB_E_INVAL, "%s: negative group stride", what);
    if (m->row_stride > ((int64_t)1 << 40) || m->group_stride > ((int64_t)1 << 46))
        return set_error(MALIB_E_INVAL, "%s: stride too large", what);
    if (output && groups_overlap(*m, rows, cols, groups))
        return set_error(MALIB_E_INVAL, "%s: the groups overlap", what);
    return MALIB_OK;
}

MatArg arg(const malib_mat* m)
{
    return m ? MatArg{m->ptr, m->row_stride, m->group_stride} : MatArg{nullptr, 0, 0};
}

malib_status check_work(void* work, int64_t have, int64_t need)
{
    if (need > 0 && (!work || have < need))
        return set_error(MALIB_E_INVAL, "the workspace needs %lld bytes, got %lld",
                         (long long)need, (long long)(work ? have : 0));
    if (need > 0 && (uintptr_t)work % 16)
        return set_error(MALIB_E_INVAL, "the workspace is not aligned to 16 bytes");
    return MALIB_OK;
}

// Workgroups of one product are counted in 31 bits (the largest tile may become 128)
malib_status check_grid(const malib_linear_desc* d, const GemmPlan& p, int64_t M, int64_t N)
{
    if (p.tile == 0)
        return MALIB_OK;
    const int64_t tile = std::min(p.tile, 128);
    const int64_t mt = (M + tile - 1) / tile, nt = (N + tile - 1) / tile;
    if (mt * nt > kMaxRows / ((int64_t)d->groups * p.splits))
        return set_error(MALIB_E_UNSUPPORTED, "the layer has 2^31 tiles or more");
    return MALIB_OK;
}

// The backward pass's launches and the layout of its workspace.  dz = dy act'(z) is
// either formed while the products load it (`fused`: one launch, but every
// tile that needs a value forms it again) or once into the workspace (rows padded to
// 16 bytes).  dbias comes with dW's product (sums of what it multiplies), except
// where that is rounded or the product's tile has no room for it: then from the
// kernel that forms dz.
// Fused against apart (us): up to kFusedMost values it saves a launch, 256 x 256 -> 256
// bf16 ReLU 8.7 and 12.8, 1024 rows 12.3 and 16.8, 4096 rows 15.1 and 16.9, fp32 SiLU
// 12.4 and 16.0, 21.5 and 20.7, 28.6 and 26.4; above, 16384 rows 28.7 and 26.3, fp32 66.7
// and 56.3.  Up to kFusedWidth inputs few tiles share a value: 65536 x 64 -> 64 bf16 17.5 and
// 28.2, 128 -> 512 63 and 81, fp32 32.8 and 37.9, 221 and 224.  The rule is wrong where out is
// wide and in narrow or not a whole tile (18807 x 24 -> 5824 bf16 265 and 205, 65536 x 96
// -> 512 92 and 78, fp32 268 and 222) and for few rows of wide layers (2048 x 1024 -> 512 bf16
// 31.6 and 26.4, fp32 62 and 50).
struct BackwardPlan {
    GemmPlan dx, dw;
    DzPlan dz;
    bool fused, own_sums;   // own_sums: dbias from dz's kernel
    int64_t dz_ld, dz_at, sum_at, dw_at, dx_at, bytes;
};

BackwardPlan make_backward_plan(const malib_linear_desc* d)
{
    const int size = type_size(d->dtype), ch = 16 / size;
    const bool act = d->act != MALIB_ACT_NONE;
    const bool rounded = size == 2 && (d->act == MALIB_ACT_GELU || d->act == MALIB_ACT_SILU);
    BackwardPlan p;
    p.dz = dz_plan(d->groups, d->rows, d->out, size);
    p.fused = act && !rounded &&
              (d->groups * d->rows * d->out <= kFusedMost || d->in <= kFusedWidth);
    // (dz formed in the workspace has padded rows)
    int loads = loads_of(d->in, size);
    if (!act || p.fused)
        loads = std::max(loads, loads_of(d->out, size));
    if (p.fused)
        loads = std::max<int>(loads, kLoadsStaged);
    backward_plans(d->groups, d->rows, d->in, d->out, size, loads, p.dw, p.dx);
    p.own_sums = (act && !p.fused) || p.dw.tile == 256;
    p.dz_ld = (d->out + ch - 1) / ch * ch;
    p.dz_at = 0;
    p.sum_at = act && !p.fused ? align256(d->groups * d->rows * p.dz_ld * (int64_t)size) : 0;
    p.dw_at = p.sum_at + align256(std::max(p.dz.sum_bytes, p.dw.sum_bytes));
    p.dx_at = p.dw_at + align256(p.dw.part_bytes);
    p.bytes = p.dx_at + align256(p.dx.part_bytes);
    return p;
}

// The plan of a description: a few microseconds of the host to make, so each thread
// keeps the last ones (it depends on nothing else).
const BackwardPlan& backward_plan(const malib_linear_desc* d)
{
    struct Kept {
        malib_linear_desc d;
        BackwardPlan p;
    };
    constexpr uint64_t kSlots = 32;
    static thread_local Kept kept[kSlots];   // (no description has groups = 0)
    const uint64_t h = (uint64_t)d->rows * 31 + (uint64_t)d->in * 17 + (uint64_t)d->out * 7 +
                       (uint64_t)d->groups * 3 + (uint64_t)(d->act + 4 * d->dtype);
    Kept& k = kept[h * 0x9E3779B97F4A7C15ull >> 59];
    static_assert(kSlots == 1u << (64 - 59), "");
    static_assert(sizeof(malib_linear_desc) == 40, "no padding: compared as bytes");
    if (std::memcmp(&k.d, d, sizeof *d) != 0) {
        k.p = make_backward_plan(d);
        k.d = *d;
    }
    return k.p;
}

}  // namespace

extern "C" {

malib_status malib_linear_work(const malib_linear_desc* d, int32_t backward, int64_t* work_bytes)
{
    TRY(check_linear(d));
    if (!work_bytes)
        return set_error(MALIB_E_INVAL, "work_bytes is NULL");
    *work_bytes = backward ? backward_plan(d).bytes
                           : linear_plan(d->groups, d->rows, d->out, d->in, type_size(d->dtype))
                                 .part_bytes;
    return MALIB_OK;
}

malib_status malib_linear(const malib_linear_desc* d, const malib_mat* x, const malib_mat* w,
                          const float* bias, const malib_mat* residual, const malib_mat* pre,
                          const malib_mat* y, void* work, int64_t work_bytes, void* stream)
{
    TRY(check_linear(d));
    if (d->rows == 0)
        return MALIB_OK;
    const int size = type_size(d->dtype);
    TRY(check_mat(x, "x", d->rows, d->in, d->groups, size, false));
    TRY(check_mat(w, "w", d->out, d->in, d->groups, size, false));
    TRY(check_mat(y, "y", d->rows, d->out, d->groups, size, true));
    if (residual)
        TRY(check_mat(residual, "residual", d->rows, d->out, d->groups, size, false));
    if (pre)
        TRY(check_mat(pre, "pre", d->rows, d->out, d->groups, size, true));
    if (bias && (uintptr_t)bias % 4)
        return set_error(MALIB_E_INVAL, "bias is not aligned to its elements");
    const GemmPlan p = linear_plan(d->groups, d->rows, d->out, d->in, size);
    TRY(check_grid(d, p, d->rows, d->out));
    TRY(check_work(work, work_bytes, p.part_bytes));
    GemmArgs a{};
    a.a = arg(x);
    a.b = arg(w);
    a.c = arg(y);
    a.res = arg(residual);
    a.pre = arg(pre);
    a.bias = bias;
    a.M = (int)d->rows;
    a.N = (int)d->out;
    a.K = (int)d->in;
    a.groups = (int)d->groups;
    a.act = d->act;
    HIP_TRY(launch_linear(d->dtype, a, p, (float*)work, (hipStream_t)stream));
    return MALIB_OK;
}

malib_status malib_linear_backward(const malib_linear_desc* d, const malib_mat* dy,
                                   const malib_mat* x, const malib_mat* w, const malib_mat* pre,
                                   const malib_mat* dx, const malib_mat* dw, float* dbias,
                                   void* work, int64_t work_bytes, void* stream)
{
    TRY(check_linear(d));
    const int size = type_size(d->dtype);
    const bool act = d->act != MALIB_ACT_NONE;
    if (d->rows > 0) {   // without rows the inputs may be empty: only sums of nothing are written
        TRY(check_mat(dy, "dy", d->rows, d->out, d->groups, size, false));
        if (act)
            TRY(check_mat(pre, "pre", d->rows, d->out, d->groups, size, false));
        if (dw)
            TRY(check_mat(x, "x", d->rows, d->in, d->groups, size, false));
        if (dx) {
            TRY(check_mat(w, "w", d->out, d->in, d->groups, size, false));
            TRY(check_mat(dx, "dx", d->rows, d->in, d->groups, size, true));
        }
    }
    if (dw)
        TRY(check_mat(dw, "dw", d->out, d->in, d->groups, size, true));
    if (dbias && (uintptr_t)dbias % 4)
        return set_error(MALIB_E_INVAL, "dbias is not aligned to its elements");
    const BackwardPlan& p = backward_plan(d);
    if (dx)
        TRY(check_grid(d, p.dx, d->rows, d->in));
    if (dw)
        TRY(check_grid(d, p.dw, d->out, d->in));
    TRY(check_work(work, work_bytes, p.bytes));
    hipStream_t s = (hipStream_t)stream;
    char* ws = (char*)work;
    const bool rows = d->rows > 0;
    MatArg dz = rows ? arg(dy) : MatArg{nullptr, d->out, 0};
    const bool products = dw || (dx && rows);
    const bool make_dz = act && !p.fused && products && rows;
    const bool own_sums = dbias && (p.own_sums || !dw);
    DbArgs db{};
    if (make_dz || own_sums) {
        MatArg to{nullptr, 0, 0};
        if (make_dz)
            to = MatArg{ws + p.dz_at, p.dz_ld, d->rows * p.dz_ld};
        float* sums = !own_sums ? nullptr : p.dz.parts > 1 ? (float*)(ws + p.sum_at) : dbias;
        HIP_TRY(launch_dz(d->dtype, p.dz, arg(dy), arg(pre), to, d->act, (int)d->groups,
                          (int)d->rows, (int)d->out, sums, s));
        if (sums && p.dz.parts > 1)
            db = DbArgs{sums, d->groups * d->out, p.dz.parts, dbias};
        if (make_dz)
            dz = to;
    }
    GemmArgs ax{}, aw{};
    ax.groups = aw.groups = (int)d->groups;
    ax.a = aw.a = dz;
    ax.a_padded = aw.a_padded = make_dz;
    if (act && p.fused && rows) {
        ax.a_pre = aw.a_pre = arg(pre);
        ax.a_act = aw.a_act = d->act;
    }
    if (dx && rows) {
        ax.b = arg(w);
        ax.c = arg(dx);
        ax.M = (int)d->rows;
        ax.N = (int)d->in;
        ax.K = (int)d->out;
    }
    if (dw) {
        aw.b = rows ? arg(x) : MatArg{nullptr, d->in, 0};
        aw.c = arg(dw);
        aw.M = (int)d->out;
        aw.N = (int)d->in;
        aw.K = (int)d->rows;
        aw.sum_out = dbias && !own_sums ? dbias : nullptr;
    }
    HIP_TRY(launch_linear_backward(d->dtype, aw, p.dw, (float*)(ws + p.dw_at),
                                   (float*)(ws + p.sum_at), ax, p.dx, (float*)(ws + p.dx_at), db,
                                   s));
    return MALIB_OK;
}

static malib_status check_loss(int dtype, int64_t rows, int64_t A)
{
    if (dtype != MALIB_DT_F32 && dtype != MALIB_DT_BF16)
        return set_error(MALIB_E_INVAL, "unknown dtype %d", dtype);
    if (rows < 0 || rows > kMaxRows)
        return set_error(MALIB_E_INVAL, "rows must be in [0, 2^31)");
    if (A < 1 || A > kMaxWidth)
        return set_error(MALIB_E_INVAL, "n_actions must be in [1, 2^24]");
    return MALIB_OK;
}

// A [rows][A] buffer of the losses.
static malib_status check_rows(const void* p, int64_t stride, const char* what, int64_t rows,
                               int64_t A, int size, bool output)
{
    if ((uintptr_t)p % size)
        return set_error(MALIB_E_INVAL, "%s is not aligned to its elements", what);
    if (rows > 1 && (stride < (output ? A : 0) || stride > ((int64_t)1 << 40)))
        return set_error(MALIB_E_INVAL, "%s: bad row stride %lld for %lld entries", what,
                         (long long)stride, (long long)A);
    return MALIB_OK;
}

malib_status malib_loss_work(int32_t dtype, int64_t rows, int64_t A, int64_t* work_bytes)
{
    TRY(check_loss(dtype, rows, A));
    if (!work_bytes)
        return set_error(MALIB_E_INVAL, "work_bytes is NULL");
    // (of lists that as many threads take, the longest needs the most workgroups)
    *work_bytes = 0;
    for (const int top : {0, 32, 64, 128, 256})
        *work_bytes = std::max(*work_bytes, loss_plan(rows, A, top, type_size(dtype)).work_bytes);
    return MALIB_OK;
}

malib_status malib_policy_loss(const malib_policy_loss_desc* d, const void* logits,
                               const void* actions, const float* old_logp,
                               const float* advantage, const float* ref_logp,
                               const void* ref_logits, const uint8_t* mask, const float* weight,
                               float* total, float* stats, void* dlogits, void* work,
                               int64_t work_bytes, void* stream)
{
    if (!d)
        return set_error(MALIB_E_INVAL, "desc is NULL");
    TRY(check_loss(d->dtype, d->rows, d->n_actions));
    if (d->action_bytes != 1 && d->action_bytes != 4 && d->action_bytes != 8)
        return set_error(MALIB_E_INVAL, "action_bytes must be 1, 4 or 8");
    if (!(d->clip_low >= 0.0f) || !(d->clip_high >= 0.0f))
        return set_error(MALIB_E_INVAL, "clip_low and clip_high must be >= 0");
    if (!std::isfinite(d->kl_coef) || !std::isfinite(d->entropy_coef))
        return set_error(MALIB_E_INVAL, "kl_coef and entropy_coef must be finite");
    if (ref_logp && ref_logits)
        return set_error(MALIB_E_INVAL, "ref_logp and ref_logits exclude each other");
    if (d->kl_coef != 0.0f && d->rows > 0 && !ref_logp && !ref_logits)   // (of no rows: NULL)
        return set_error(MALIB_E_INVAL, "kl_coef needs ref_logp or ref_logits");
    const int size = type_size(d->dtype);
    const LossPlan p = loss_plan(d->rows, d->n_actions, 0, size);
    if (d->rows > 0) {
        if (!logits || !actions || !old_logp || !advantage)
            return set_error(MALIB_E_INVAL,
                             "logits, actions, old_logp and advantage must not be NULL");
        if ((uintptr_t)actions % d->action_bytes)
            return set_error(MALIB_E_INVAL, "actions is not aligned to its elements");
        TRY(check_rows(logits, d->logits_stride, "logits", d->rows, d->n_actions, size, false));
        if (ref_logits)
            TRY(check_rows(ref_logits, d->ref_stride, "ref_logits", d->rows, d->n_actions, size,
                           false));
        if (mask)
            TRY(check_rows(mask, d->mask_stride, "mask", d->rows, d->n_actions, 1, false));
        if (dlogits)
            TRY(check_rows(dlogits, d->dlogits_stride, "dlogits", d->rows, d->n_actions, size,
                           true));
        TRY(check_work(work, work_bytes, p.work_bytes));
    }
    LossArgs a{};
    a.logits = logits;
    a.ref_logits = ref_logits;
    a.mask = mask;
    a.weight = weight;
    a.actions = actions;
    a.old_logp = old_logp;
    a.advantage = advantage;
    a.ref_logp = ref_logp;
    a.dlogits = dlogits;
    a.stats = stats;
    a.total = total;
    a.rows = d->rows;
    a.logits_ld = d->logits_stride;
    a.ref_ld = d->ref_stride;
    a.mask_ld = d->mask_stride;
    a.dlogits_ld = d->dlogits_stride;
    a.A = (int)d->n_actions;
    a.action_bytes = d->action_bytes;
    a.row_weight = d->rows > 0 ? (float)(1.0 / (double)d->rows) : 0.0f;
    a.clip_low = d->clip_low;
    a.clip_high = d->clip_high;
    a.kl_coef = d->kl_coef;
    a.entropy_coef = d->entropy_coef;
    a.temperature = 1.0f;
    HIP_TRY(launch_loss(a, d->dtype, false, p, work, (hipStream_t)stream));
    return MALIB_OK;
}

malib_status malib_distill_loss(const malib_distill_desc* d, const void* logits,
                                const int32_t* teacher_idx, const float* teacher_logits,
                                const uint8_t* mask, const float* weight, float* total,
                                float* loss, void* dlogits, void* work, int64_t work_bytes,
                                void* stream)
{
    if (!d)
        return set_error(MALIB_E_INVAL, "desc is NULL");
    TRY(check_loss(d->dtype, d->rows, d->n_actions));
    if (d->top < 1 || d->top > 256)
        return set_error(MALIB_E_INVAL, "top must be in [1, 256]");
    if (!(d->temperature > 0.0f) || !std::isfinite(d->temperature))
        return set_error(MALIB_E_INVAL, "temperature must be positive and finite");
    const int size = type_size(d->dtype);
    const LossPlan p = loss_plan(d->rows, d->n_actions, d->top, size);
    if (d->rows > 0) {
        if (!logits || !teacher_idx || !teacher_logits)
            return set_error(MALIB_E_INVAL,
                             "logits, teacher_idx and teacher_logits must not be NULL");
        TRY(check_rows(logits, d->logits_stride, "logits", d->rows, d->n_actions, size, false));
        if (mask)
            TRY(check_rows(mask, d->mask_stride, "mask", d->rows, d->n_actions, 1, false));
        if (dlogits)
            TRY(check_rows(dlogits, d->dlogits_stride, "dlogits", d->rows, d->n_actions, size,
                           true));
        TRY(check_work(work, work_bytes, p.work_bytes));
    }
    LossArgs a{};
    a.logits = logits;
    a.mask = mask;
    a.weight = weight;
    a.idx = teacher_idx;
    a.val = teacher_logits;
    a.dlogits = dlogits;
    a.stats = loss;
    a.total = total;
    a.rows = d->rows;
    a.logits_ld = d->logits_stride;
    a.mask_ld = d->mask_stride;
    a.dlogits_ld = d->dlogits_stride;
    a.A = (int)d->n_actions;
    a.top = d->top;
    a.row_weight = d->rows > 0 ? (float)(1.0 / (double)d->rows) : 0.0f;
    a.temperature = d->temperature;
    HIP_TRY(launch_loss(a, d->dtype, true, p, work, (hipStream_t)stream));
    return MALIB_OK;
}

static malib_status check_log_probs(const malib_log_probs_desc* d)
{
    if (!d)
        return set_error(MALIB_E_INVAL, "desc is NULL");
    TRY(check_loss(d->dtype, d->rows, d->n_actions));
    if (!(d->temperature >= 0x1p-100f && d->temperature <= 0x1p100f))   // (1 / T is taken)
        return set_error(MALIB_E_INVAL, "temperature must be in [2^-100, 2^100]");
    return MALIB_OK;
}

// Actions of either direction, and what both take of logits and mask.
static malib_status check_scored(const malib_log_probs_desc* d, const void* logits,
                                 const void* actions, const uint8_t* mask)
{
    if (!logits)
        return set_error(MALIB_E_INVAL, "logits is NULL");
    TRY(check_rows(logits, d->logits_stride, "logits", d->rows, d->n_actions,
                   type_size(d->dtype), false));
    if (mask)
        TRY(check_rows(mask, d->mask_stride, "mask", d->rows, d->n_actions, 1, false));
    if (actions) {
        if (d->action_bytes != 1 && d->action_bytes != 4 && d->action_bytes != 8)
            return set_error(MALIB_E_INVAL, "action_bytes must be 1, 4 or 8");
        if ((uintptr_t)actions % d->action_bytes)
            return set_error(MALIB_E_INVAL, "actions is not aligned to its elements");
    }
    return MALIB_OK;
}

static LogpArgs logp_args(const malib_log_probs_desc* d, const void* logits, const void* actions,
                          const uint8_t* mask, const float* stats)
{
    LogpArgs a{};
    a.logits = logits;
    a.actions = actions;
    a.mask = mask;
    a.stats = const_cast<float*>(stats);
    a.rows = d->rows;
    a.logits_ld = d->logits_stride;
    a.mask_ld = d->mask_stride;
    a.dlogits_ld = d->dlogits_stride;
    a.A = (int)d->n_actions;
    a.action_bytes = d->action_bytes;
    a.temperature = d->temperature;
    return a;
}

static malib_status check_aligned(const void* p, const char* what, int bytes)
{
    if ((uintptr_t)p % bytes)
        return set_error(MALIB_E_INVAL, "%s is not aligned to %d bytes", what, bytes);
    return MALIB_OK;
}

static malib_status check_top(int32_t top)
{
    if (top < 0 || top > 256)
        return set_error(MALIB_E_INVAL, "top must be in [0, 256]");
    return MALIB_OK;
}

malib_status malib_log_probs_work(int32_t dtype, int64_t rows, int64_t A, int32_t top,
                                  int64_t* work_bytes)
{
    TRY(check_loss(dtype, rows, A));
    TRY(check_top(top));
    if (!work_bytes)
        return set_error(MALIB_E_INVAL, "work_bytes is NULL");
    *work_bytes = logp_plan(rows, A, top, type_size(dtype)).work_bytes;
    return MALIB_OK;
}

malib_status malib_log_probs(const malib_log_probs_desc* d, const void* logits,
                             const void* actions, const uint8_t* mask, float* stats,
                             int32_t* top_idx, float* top_logp, void* work, int64_t work_bytes,
                             void* stream)
{
    TRY(check_log_probs(d));
    TRY(check_top(d->top));
    if (d->rows == 0)
        return MALIB_OK;
    TRY(check_scored(d, logits, actions, mask));
    if (!stats)
        return set_error(MALIB_E_INVAL, "stats is NULL");
    if (d->top > 0 && (!top_idx || !top_logp))
        return set_error(MALIB_E_INVAL, "top_idx and top_logp must not be NULL");
    TRY(check_aligned(stats, "stats", 4));
    TRY(check_aligned(top_idx, "top_idx", 4));
    TRY(check_aligned(top_logp, "top_logp", 4));
    const LogpPlan p = logp_plan(d->rows, d->n_actions, d->top, type_size(d->dtype));
    TRY(check_work(work, work_bytes, p.work_bytes));
    LogpArgs a = logp_args(d, logits, actions, mask, stats);
    a.top = d->top;
    a.top_idx = top_idx;
    a.top_logp = top_logp;
    HIP_TRY(launch_logp(a, d->dtype, p, work, (hipStream_t)stream));
    return MALIB_OK;
}

malib_status malib_log_probs_backward(const malib_log_probs_desc* d, const void* logits,
                                      const void* actions, const uint8_t* mask,
                                      const float* stats, const float* dlogp,
                                      const float* dentropy, void* dlogits, void* stream)
{
    TRY(check_log_probs(d));
    if (d->rows == 0)
        return MALIB_OK;
    TRY(check_scored(d, logits, actions, mask));
    if (!stats || !dlogits)
        return set_error(MALIB_E_INVAL, "stats and dlogits must not be NULL");
    if (dlogp && !actions)
        return set_error(MALIB_E_INVAL, "dlogp needs actions");
    TRY(check_aligned(stats, "stats", 4));
    TRY(check_aligned(dlogp, "dlogp", 4));
    TRY(check_aligned(dentropy, "dentropy", 4));
    TRY(check_rows(dlogits, d->dlogits_stride, "dlogits", d->rows, d->n_actions,
                   type_size(d->dtype), true));
    LogpArgs a = logp_args(d, logits, actions, mask, stats);
    a.dlogp = dlogp;
    a.dentropy = dentropy;
    a.dlogits = dlogits;
    HIP_TRY(launch_logp_grad(a, d->dtype, (hipStream_t)stream));
    return MALIB_OK;
}

malib_status malib_dropout(const malib_dropout_desc* d, const void* x, const void* residual,
                           const int64_t* device_step, void* y, void* stream)
{
    if (!d)
        return set_error(MALIB_E_INVAL, "desc is NULL");
    if (d->dtype != MALIB_DT_F32 && d->dtype != MALIB_DT_BF16)
        return set_error(MALIB_E_INVAL, "unknown dtype %d", d->dtype);
    if (d->rows < 0 || d->rows > kMaxRows)
        return set_error(MALIB_E_INVAL, "rows must be in [0, 2^31)");
    if (d->cols < 1 || d->cols > kMaxWidth)
        return set_error(MALIB_E_INVAL, "cols must be in [1, 2^24]");
    if (!(d->p >= 0.0 && d->p <= 1.0))
        return set_error(MALIB_E_INVAL, "p must be in [0, 1]");
    if (d->rows == 0)
        return MALIB_OK;
    const int size = type_size(d->dtype);
    if (!x || !y)
        return set_error(MALIB_E_INVAL, "x and y must not be NULL");
    TRY(check_rows(x, d->x_stride, "x", d->rows, d->cols, size, false));
    TRY(check_rows(y, d->y_stride, "y", d->rows, d->cols, size, true));
    if (residual)
        TRY(check_rows(residual, d->residual_stride, "residual", d->rows, d->cols, size, false));
    TRY(check_aligned(device_step, "device_step", 8));
    DropoutArgs a{};
    a.x = x;
    a.residual = residual;
    a.y = y;
    a.device_step = device_step;
    a.rows = d->rows;
    a.cols = d->cols;
    a.x_ld = d->x_stride;
    a.residual_ld = d->residual_stride;
    a.y_ld = d->y_stride;
    a.seed = d->seed;
    a.step = d->step;
    a.layer = d->layer;
    a.drop = (uint32_t)std::llrint(d->p * 65536.0);
    a.scale = a.drop < 65536u ? (float)(65536.0 / (65536.0 - a.drop)) : 0.0f;
    HIP_TRY(launch_dropout(a, d->dtype, (hipStream_t)stream));
    return MALIB_OK;
}

static malib_status check_fp4(const malib_fp4_desc* d)
{
    if (!d)
        return set_error(MALIB_E_INVAL, "desc is NULL");
    const malib_linear_desc l{d->dtype, d->act, d->groups, d->rows, d->in, d->out};
    TRY(check_linear(&l));
    if (d->groups * d->out > kMaxValues / d->in)
        return set_error(MALIB_E_UNSUPPORTED, "groups * out * in must be at most 2^46");
    if (d->scale_group != 32 && d->scale_group != 64 && d->scale_group != 128)
        return set_error(MALIB_E_INVAL, "scale_group must be 32, 64 or 128");
    if (d->reserved != 0)
        return set_error(MALIB_E_INVAL, "reserved must be 0");
    return MALIB_OK;
}

static malib_status check_codes(const void* codes, const void* scales)
{
    if (!codes || !scales)
        return set_error(MALIB_E_INVAL, "codes and scales must not be NULL");
    TRY(check_aligned(codes, "codes", 16));
    return check_aligned(scales, "scales", 8);
}

static Fp4Args fp4_args(const malib_fp4_desc* d, const uint8_t* codes, const uint16_t* scales)
{
    Fp4Args a{};
    a.codes = const_cast<uint8_t*>(codes);
    a.scales = const_cast<uint16_t*>(scales);
    a.groups = (int)d->groups;
    a.M = (int)d->rows;
    a.N = (int)d->out;
    a.K = (int)d->in;
    a.scale_group = d->scale_group;
    a.act = d->act;
    a.tiles = (a.N + 15) / 16;
    a.blocks_k = (a.K + 127) / 128;
    return a;
}

malib_status malib_quantize_fp4(const malib_fp4_desc* d, const malib_mat* w, uint8_t* codes,
                                uint16_t* scales, void* stream)
{
    TRY(check_fp4(d));
    TRY(check_mat(w, "w", d->out, d->in, d->groups, type_size(d->dtype), false));
    TRY(check_codes(codes, scales));
    Fp4Args a = fp4_args(d, codes, scales);
    a.w = arg(w);
    HIP_TRY(launch_quantize_fp4(a, d->dtype, (hipStream_t)stream));
    return MALIB_OK;
}

malib_status malib_dequantize_fp4(const malib_fp4_desc* d, const uint8_t* codes,
                                  const uint16_t* scales, const malib_mat* w, void* stream)
{
    TRY(check_fp4(d));
    TRY(check_codes(codes, scales));
    TRY(check_mat(w, "w", d->out, d->in, d->groups, type_size(d->dtype), true));
    Fp4Args a = fp4_args(d, codes, scales);
    a.w = arg(w);
    HIP_TRY(launch_dequantize_fp4(a, d->dtype, (hipStream_t)stream));
    return MALIB_OK;
}

malib_status malib_linear_fp4(const malib_fp4_desc* d, const malib_mat* x,
                              const uint8_t* codes, const uint16_t* scales, const float* bias,
                              const malib_mat* residual, const malib_mat* y, void* stream)
{
    TRY(check_fp4(d));
    if (d->rows == 0)
        return MALIB_OK;
    const int size = type_size(d->dtype);
    TRY(check_mat(x, "x", d->rows, d->in, d->groups, size, false));
    TRY(check_codes(codes, scales));
    TRY(check_mat(y, "y", d->rows, d->out, d->groups, size, true));
    if (residual)
        TRY(check_mat(residual, "residual", d->rows, d->out, d->groups, size, false));
    TRY(check_aligned(bias, "bias", 4));
    Fp4Args a = fp4_args(d, codes, scales);
    a.x = arg(x);
    a.res = arg(residual);
    a.y = arg(y);
    a.bias = bias;
    const Fp4Plan p = fp4_plan(d->groups, d->rows, d->out, d->in, size);
    HIP_TRY(launch_linear_fp4(a, d->dtype, p, (hipStream_t)stream));
    return MALIB_OK;
}

}  // extern "C"
