// Host side of the gated block Y = (act(X Wg) * (X Wu)) Wd: arguments, workspace, order of the launches; the kernel that copies matrices
// whose rows cannot be read in pieces of 16 bytes.
#include "../../include/bmgd.h"
#include "bmgd_internal.h"
#include "gated_internal.h"

#include <stdio.h>

#include <algorithm>
#include <atomic>
#include <new>

using namespace bmgd;

namespace {

constexpr int64_t kMaxWidth = int64_t(1) << 20;
constexpr int64_t kMaxRows = (int64_t(1) << 30) - 1;

int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

struct Layout {
    size_t h, d, x, gate, up, down, dy, partial, counter, zeros, scaled, scale_h, scale_d, total;
};

bool valid(const bmgd_gated_config& c, const char** why)
{
    if (c.p < 1 || c.hidden < 1 || c.out_n < 1 || c.p > kMaxWidth || c.hidden > kMaxWidth || c.out_n > kMaxWidth)
        *why = "p, hidden and out_n must be in [1, 2^20]";
    else if (c.max_rows < 1 || c.max_rows > kMaxRows) *why = "max_rows must be in [1, 2^30)";
    else if (c.dtype != BMGD_BF16 && c.dtype != BMGD_F16) *why = "dtype must be BMGD_BF16 or BMGD_F16";
    else if (c.activation != BMGD_ACT_SILU && c.activation != BMGD_ACT_GELU && c.activation != BMGD_ACT_RELU) *why = "unknown activation";
    else if ((c.max_rows / 64 + 1) * (2 * std::max(c.p, std::max(c.hidden, c.out_n)) / 64 + 2) >= (int64_t(1) << 30) ||
             (c.p / 64 + 1) * (2 * c.hidden / 64 + 2) >= (int64_t(1) << 30) || (c.hidden / 64 + 1) * (c.out_n / 64 + 1) >= (int64_t(1) << 30))
        *why = "a product has 2^30 tiles of 64 x 64 or more";
    else return true;
    return false;
}

Layout make_layout(const bmgd_gated_config& c)
{
    Layout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t r = at; at += (bytes + 255) / 256 * 256; return r; };
    const size_t r = (size_t)c.max_rows, f64 = (size_t)up(c.hidden, 64), f8 = (size_t)up(c.hidden, 8), p8 = (size_t)up(c.p, 8), c8 = (size_t)up(c.out_n, 8);
    const size_t rows_between = std::max(r, 2 * std::min(r, (size_t)kGatedPairRows));
    l.h = take(2 * rows_between * f64);
    l.d = take(4 * rows_between * f64);
    l.x = take(2 * r * p8);
    l.gate = take(2 * (size_t)c.p * f8);
    l.up = take(2 * (size_t)c.p * f8);
    l.down = take(2 * (size_t)c.hidden * c8);
    l.dy = take(2 * r * c8);
    l.partial = take(kGatedPartialBytes);
    l.counter = take(kGatedCounters * sizeof(unsigned));
    l.zeros = take(256);
    if (c.dtype == BMGD_F16) {
        l.scaled = take(256);
        l.scale_h = take(rows_between * f64 / 8);
        l.scale_d = take(2 * rows_between * f64 / 8);
    }
    l.total = at;
    return l;
}

int fail_static(int code, const char* call, const char* msg)
{
    char buf[256];
    snprintf(buf, sizeof buf, "%s: %s", call, msg);
    set_create_error(buf);
    return code;
}

struct PackArgs { GatedPack q; };

// A thread moves eight elements, from any even address (one instruction all the same) to 16-byte aligned ones.
__global__ void __launch_bounds__(256) gated_pack_kernel(PackArgs args)
{
    typedef unsigned short ushort8 __attribute__((ext_vector_type(8)));
    typedef unsigned short ushort8u __attribute__((ext_vector_type(8), aligned(2)));
    const GatedPack::One m = args.q.m[blockIdx.y];
    const int64_t per_row = m.to_ld >> 3, pieces = m.rows * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t r = pieces >> 31 ? i / per_row : (int64_t)((unsigned)i / (unsigned)per_row), c = 8 * (i - r * per_row);
        const unsigned short* from = m.from + r * m.from_ld + c;
        ushort8 v;
        if (c + 8 <= m.cols) {
            v = *(const ushort8u*)from;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = c + k < m.cols ? from[k] : (unsigned short)0;
        }
        *(ushort8*)(m.to + r * m.to_ld + c) = v;
    }
}

}  // namespace

struct bmgd_gated {
    bmgd_gated_config cfg;
    Layout lay;
    int device = 0, num_cus = 0;
    char* base = nullptr;
    bool owned = false, used = false, captured = false;        // `used`: by calls that were not captured into a graph
    hipStream_t last = nullptr;             // of the last such call
    hipEvent_t order = nullptr;
    char err[256] = "";
    int turn = 0;                           // of calls in f16, see GatedProduct
    int tile = -1, shares = 0;              // asked for by tests
    bool wide = false;                      // every row has eight elements or more, as loose tiles want them
    struct Kept { int64_t rows = -1; int what = 0; bmgd::GatedCut cut[3]; } kept[32];      // by rows modulo 8 and launch, see plan()
};

namespace bmgd {

static int64_t columns_of(const GatedProduct& q, GatedOp op)
{
    return op == kOpUp ? 2 * q.half : op == kOpDown ? q.half : op == kOpWeight && q.half ? 2 * q.half : q.N;
}
static int64_t steps_of(const GatedProduct& q, GatedOp op) { return ((op == kOpInput ? 2 * q.half : q.K) + kGatedStep - 1) / kGatedStep; }

hipError_t gated_launch_pack(const GatedPack& q, hipStream_t stream)
{
    int64_t most = 1;
    for (int i = 0; i < q.count; ++i) most = std::max(most, q.m[i].rows * (q.m[i].to_ld >> 3));
    const unsigned blocks = (unsigned)std::min<int64_t>((most + 255) / 256, 4096);
    PackArgs a{q};
    hipLaunchKernelGGL(gated_pack_kernel, dim3(blocks, (unsigned)q.count), dim3(256), 0, stream, a);
    return hipGetLastError();
}

// The time of a launch, in us, as measured for 123 shapes of one to 8,192 rows and widths of 64 to 8,192 in every product, tile and split, weights not in
// any cache (13,971 launches; near the fastest ones of a shape the formula is off by 18 % in the mean square, and its choice is 3 % slower than the fastest):
//      base + max(rounds (steps lat + once), workgroups of a unit (steps thr + leave), bytes / rate) + join
// with the steps of a workgroup, the rounds that the units need for all workgroups, a rate that takes enough bytes on their way (2.2 us from request to
// arrival), and where workgroups share tiles
//      join = join + each splits + megabytes of parts per unit write.
// It does not know where rows begin: kOpDown, which reads G and U on its way out, takes half as long again where theirs begin at odd places (1,000 rows, p = 512, hidden 2,731,
// out 1,000: 23 us, by the formula 15).  Nothing but sizes counts, not what is at hand or wanted besides: Y has the same bits whether G and U are kept or not.
void gated_plan(GatedProduct* const* qs, const GatedOp* ops, int count, int num_cus, int asked_tile, int64_t asked)
{
    struct Cost { int bm, bn, per_cu, ahead; double lat, thr, once[3], leave[3], join, each, write; };       // [kOpUp, kOpDown, the others]
    static const Cost cost[kTiles] = {
        {256, 256, 1, 1, 1.38, 1.45, {7.0, 25.6, 13.4}, {8.7, 8.1, 2.6}, 0.55, 0.4, 117.0}, {128, 128, 2, 1, 0.29, 0.58, {1.3, 3.2, 2.95}, {1.15, 3.0, 1.45}, 0.05, 0.53, 122.0},
        {128, 128, 1, 2, 0.56, 0.36, {1.5, 4.5, 2.75}, {1.45, 1.15, 0.55}, 0.0, 0.32, 111.0},
        {64, 64, 3, 2, 0.01, 0.27, {0.85, 0.35, 2.35}, {0.6, 0.65, 0.45}, 0.95, 0.37, 40.0}, {32, 128, 2, 3, 0.05, 0.55, {1.3, 2.2, 0.3}, {0.7, 1.5, 0.0}, 0.8, 0.5, 60.0},
        {16, 128, 2, 3, 0.41, 0.46, {0.8, 1.05, 0.0}, {0.8, 1.7, 0.1}, 1.2, 0.28, 60.0}};
    constexpr double kBase = 2.8;                              // a launch that does nothing
    constexpr double kBytesPerUs = 4.4e6, kTripUs = 2.2;
    double best = 1e300;
    for (int t = 0; t < kTiles; ++t) {
        if (asked_tile >= 0 && t != asked_tile) continue;
        const Cost& k = cost[t];
        bool fits = true;
        int64_t most_steps = 1;
        double bytes = 0.0;
        for (int i = 0; i < count; ++i) {
            const GatedProduct& q = *qs[i];
            fits = fits && !(t >= kTile32 && (count > 1 || ops[i] > kOpDown || q.M > k.bm)) && !(q.pair && (ops[i] == kOpUp || ops[i] == kOpDown) && k.bm > 64);
            most_steps = std::max(most_steps, steps_of(q, ops[i]));
            const double M = (double)q.M, N = (double)columns_of(q, ops[i]), K = (double)steps_of(q, ops[i]) * kGatedStep;
            bytes += 2.0 * (M * K + K * N + M * N);
        }
        if (!fits) continue;
        for (int64_t want = asked_tile >= 0 ? asked : 1; want <= 64; want += asked_tile >= 0 ? 64 : want < 4 ? 1 : want / 2) {
            struct { int64_t tm, tn, splits, per; } plan[3];
            const int64_t target = (most_steps + want - 1) / want;
            int64_t groups = 0, counters = 0;
            size_t parts = 0;
            double longest = 0.0, work = 0.0, sum = 0.0, most_splits = 0.0;
            bool ok = want == 1 || target >= 2;
            for (int i = 0; i < count && ok; ++i) {
                const GatedProduct& q = *qs[i];
                const int64_t steps = steps_of(q, ops[i]), tm = (q.M + k.bm - 1) / k.bm, tn = (columns_of(q, ops[i]) + k.bn - 1) / k.bn, tiles = tm * tn;
                const int64_t shares = std::max<int64_t>(1, (steps + target - 1) / target), per = std::max<int64_t>(1, (steps + shares - 1) / shares);
                const int64_t splits = std::max<int64_t>(1, (steps + per - 1) / per);
                if (tiles >= (int64_t(1) << 28)) { ok = false; break; }
                plan[i] = {tm, tn, splits, per};
                groups += tiles * splits;
                if (splits > 1) {
                    counters += tiles;
                    parts += (size_t)(tiles * splits) * k.bm * k.bn * 4;
                    most_splits = std::max(most_splits, (double)splits);
                }
                const int kind = ops[i] == kOpUp ? 0 : ops[i] == kOpDown ? 1 : 2;
                const double turn = per * k.lat + k.once[kind], share = per * k.thr + k.leave[kind];
                longest = std::max(longest, std::max(turn, share));
                sum += (double)(tiles * splits) * turn;
                work += (double)(tiles * splits) * share;
            }
            if (!ok || counters > kGatedCounters || parts > kGatedPartialBytes) break;
            const int64_t of_unit = (groups + num_cus - 1) / num_cus, rounds = (of_unit + k.per_cu - 1) / k.per_cu;
            const double in_turn = longest + (double)(rounds - 1) * sum / (double)groups, together = work / (double)groups * (double)of_unit;
            const double on_way = (double)std::min<int64_t>(groups, (int64_t)num_cus * k.per_cu) * k.ahead * (k.bm + k.bn) * 2 * kGatedStep;
            double us = kBase + std::max(std::max(in_turn, together), bytes / std::min(kBytesPerUs, on_way / kTripUs));
            if (parts) us += k.join + k.each * most_splits + k.write * 1e-6 * (double)parts / num_cus;
            if (us < best) {
                best = us;
                size_t at = 0;
                int counter = 0;
                for (int i = 0; i < count; ++i) {
                    GatedProduct& q = *qs[i];
                    q.tile = t;
                    q.us = us;
                    q.tiles_m = (int)plan[i].tm;
                    q.tiles_n = (int)plan[i].tn;
                    q.splits = (int)plan[i].splits;
                    q.per_split = (int)plan[i].per;
                    q.first_part = at;
                    q.first_counter = counter;
                    if (q.splits > 1) {
                        at += (size_t)(plan[i].tm * plan[i].tn * plan[i].splits) * k.bm * k.bn;
                        counter += (int)(plan[i].tm * plan[i].tn);
                    }
                }
            }
        }
    }
    if (best == 1e300 && asked_tile >= 0) gated_plan(qs, ops, count, num_cus);
}

}  // namespace bmgd

namespace {

int fail(bmgd_gated* b, int code, const char* call, const char* what, const char* msg = "")
{
    snprintf(b->err, sizeof b->err, "%s: %s%s%s", call, what, *msg ? " " : "", msg);
    return code;
}

int hip_fail(bmgd_gated* b, hipError_t e, const char* what)
{
    (void)hipGetLastError();
    return fail(b, e == hipErrorOutOfMemory ? BMGD_ENOMEM : BMGD_EHIP, what, hipGetErrorString(e));
}

#define GATED_TRY(b, call)                                               \
    do {                                                                 \
        hipError_t e_ = (call);                                          \
        if (e_ != hipSuccess) return hip_fail((b), e_, #call);           \
    } while (0)

// NULL if m describes rows x cols elements that a kernel can be given.
const char* bad_matrix(const bmgd_matrix& m, int64_t rows, int64_t cols)
{
    if (rows == 0) return nullptr;
    if (!m.data) return "must not be NULL";
    if ((uintptr_t)m.data & 1) return "must be 2-byte aligned";
    if (rows > 1 && m.stride < cols) return "has rows closer together than they are long";
    if (m.stride > (int64_t(1) << 40)) return "has rows more than 2^40 elements apart";
    return nullptr;
}

struct Named {
    const char* name;
    const bmgd_matrix* m;
    int64_t rows, cols;
    bool optional;
};

int check(bmgd_gated* b, const char* call, const Named* list, int n)
{
    for (int i = 0; i < n; ++i) {
        if (list[i].optional && !list[i].m->data) continue;
        if (const char* why = bad_matrix(*list[i].m, list[i].rows, list[i].cols))
            return fail(b, BMGD_EINVAL, call, list[i].name, why);
    }
    return BMGD_OK;
}

bool direct(const bmgd_matrix& m, int64_t rows, int64_t cols) { return ((uintptr_t)m.data & 15) == 0 && cols % 8 == 0 && (rows <= 1 || m.stride % 8 == 0); }
bool pair_direct(const bmgd_matrix& m, const bmgd_matrix& m2, int64_t rows, int64_t cols)
{
    return direct(m, rows, cols) && direct(m2, rows, cols) && (rows <= 1 || m.stride == m2.stride);
}

inline int64_t unless(bool nothing, int64_t elements) { return nothing ? 0 : elements; }

// Which of a call's two launches are loose.  A loose launch takes 10 to 30 % longer (14 rows, p = 860, hidden 2,992, out 141, backward: 24.9 us for 21.7 in both), a copying
// launch 3.3 us and the time for its bytes (2.6 MB a us: 4.1 there): 100 rows, p = 200, hidden 600, out 130, backward, take 14.8 us loose and 17.0 with copies,
// 7 rows, p = 157, hidden 7,614, out 2,409, forward, 21.6 and 32.6.
struct Way { bool can; int64_t elements; double us; };         // of a launch: may it be loose, what is to copy where it is not, what it takes then
void choose(const Way& x, const Way& y, bool* loose_x, bool* loose_y)
{
    double best = 1e300;
    for (int m = 3; m >= 0; --m) {
        if (((m & 1) && !x.can) || ((m & 2) && !y.can)) continue;
        const int64_t copied = (m & 1 ? 0 : x.elements) + (m & 2 ? 0 : y.elements);
        const double us = (copied ? 3.3 + (double)copied * (2 / 2.6e6) : 0.0) + 0.2 * ((m & 1) && x.elements ? x.us : 0.0) + 0.2 * ((m & 2) && y.elements ? y.us : 0.0);
        if (us < best) {
            best = us;
            *loose_x = m & 1;
            *loose_y = m & 2;
        }
    }
}

// Operands as the kernels read them: rows of a multiple of eight elements, 16-byte aligned; a launch of loose tiles reads others too, for the rest they are
// copied to the workspace first.
struct Operands {
    bmgd_gated* b;
    GatedPack pack{};

    GatedMat copy(const bmgd_matrix& m, int64_t rows, int64_t cols, size_t area)
    {
        GatedPack::One& o = pack.m[pack.count++];
        o.from = static_cast<const unsigned short*>(m.data);
        o.to = reinterpret_cast<unsigned short*>(b->base + area);
        o.from_ld = m.stride;
        o.to_ld = up(cols, 8);
        o.rows = rows;
        o.cols = cols;
        return GatedMat{o.to, o.to_ld};
    }
    // `loose`: whether the launch may read the operand where it is, and on return whether it has to be a loose one for that
    GatedMat use(const bmgd_matrix& m, int64_t rows, int64_t cols, size_t area, bool may, bool* loose)
    {
        if (rows == 0) return GatedMat{b->base + area, up(cols, 8)};
        if (may) *loose = *loose || !direct(m, rows, cols);
        else if (!direct(m, rows, cols)) return copy(m, rows, cols, area);
        return GatedMat{m.data, rows <= 1 ? cols : m.stride};
    }
    // the two matrices that one product reads side by side: their rows are equally far apart
    void use_pair(const bmgd_matrix& m, const bmgd_matrix& m2, int64_t rows, int64_t cols, size_t area, size_t area2, bool may, bool* loose, GatedMat* o, GatedMat* o2)
    {
        const bool whole = pair_direct(m, m2, rows, cols);
        if (whole || (may && (rows <= 1 || m.stride == m2.stride))) {
            *loose = *loose || !whole;
            *o = GatedMat{m.data, rows <= 1 ? cols : m.stride};
            *o2 = GatedMat{m2.data, o->ld};
        } else {
            *o = copy(m, rows, cols, area);
            *o2 = copy(m2, rows, cols, area2);
        }
    }
};

GatedMat plain(const bmgd_matrix& m) { return GatedMat{m.data, m.stride}; }

// The block's device is current as long as this lives, then the one that was.
struct OnDevice {
    int before = -1;
    hipError_t e;
    explicit OnDevice(int device)
    {
        int current = -1;
        e = hipGetDevice(&current);
        if (e != hipSuccess || current == device) return;
        e = hipSetDevice(device);
        if (e == hipSuccess) before = current;
    }
    ~OnDevice()
    {
        if (before >= 0) (void)hipSetDevice(before);
    }
    OnDevice(const OnDevice&) = delete;
};

// Work of calls on different streams is made in the order of the calls: they share the workspace.  A call that is captured into a graph runs when the graph is
// launched: it waits for nothing outside, and is not what a later call waits for, which is still the one before it.
int enter(bmgd_gated* b, hipStream_t s)
{
    if (b->used && b->last == s) return BMGD_OK;
    hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
    GATED_TRY(b, hipStreamIsCapturing(s, &st));
    if (st != hipStreamCaptureStatusNone) {
        b->captured = true;
        return BMGD_OK;
    }
    if (b->used) {
        GATED_TRY(b, hipStreamIsCapturing(b->last, &st));
        if (st != hipStreamCaptureStatusNone)
            return fail(b, BMGD_ESTATE, "the gated block", "cannot wait for its last call: that one's stream is being captured into a graph");
        GATED_TRY(b, hipEventRecord(b->order, b->last));
        GATED_TRY(b, hipStreamWaitEvent(s, b->order, 0));
    }
    b->last = s;
    b->used = true;
    return BMGD_OK;
}

// The choice takes 1 us for a product and 2 for three, a fifth of what a call of few rows takes in all, and depends on the block's sizes and the rows alone:
// it is kept for the next call of as many rows.  `what`: the product, or 8 and a bit for each of those made in one launch.
void plan(bmgd_gated* b, GatedProduct* const* q, const GatedOp* op, int count, int64_t rows, int what)
{
    bmgd_gated::Kept& k = b->kept[(rows & 7) * 4 + (what < 8 ? what : 3)];
    const bool known = k.rows == rows && k.what == what && b->tile < 0;
    if (!known) gated_plan(q, op, count, b->num_cus, b->tile, b->shares);
    for (int i = 0; i < count; ++i) {
        if (known) static_cast<GatedCut&>(*q[i]) = k.cut[i];
        else k.cut[i] = *q[i];
        q[i]->act = b->cfg.activation;
        q[i]->partial = reinterpret_cast<float*>(b->base + b->lay.partial) + q[i]->first_part;
        q[i]->counter = reinterpret_cast<unsigned*>(b->base + b->lay.counter) + q[i]->first_counter;
        q[i]->zeros = b->base + b->lay.zeros;
    }
    k.rows = b->tile < 0 ? rows : -1;
    k.what = what;
}

void plan(bmgd_gated* b, GatedProduct& q, GatedOp op, int64_t rows)
{
    GatedProduct* one = &q;
    plan(b, &one, &op, 1, rows, op);
}

// f16: where the exponents of H and D stand, for a product that writes or reads them.
void scales(bmgd_gated* b, GatedProduct& q, size_t scale, size_t scale2 = 0)
{
    if (b->cfg.dtype != BMGD_F16) return;
    q.scale = reinterpret_cast<unsigned char*>(b->base + scale);
    q.scale2 = reinterpret_cast<unsigned char*>(b->base + scale2);
    q.scaled = reinterpret_cast<unsigned*>(b->base + b->lay.scaled);
    q.turn = b->turn;
}

int launch(bmgd_gated* b, const GatedProduct& q, GatedOp op, hipStream_t s)
{
    const hipError_t e = b->cfg.dtype == BMGD_F16 ? gated_launch_f16(q, op, s) : gated_launch_bf16(q, op, s);
    if (e != hipSuccess) return hip_fail(b, e, "launch of a product of the gated block");
    return BMGD_OK;
}

#define GATED_DO(expr)                     \
    do {                                   \
        const int rc_ = (expr);            \
        if (rc_ != BMGD_OK) return rc_;    \
    } while (0)

int forward(bmgd_gated* b, int64_t rows, const bmgd_gated_tensors& t, hipStream_t s)
{
    const bmgd_gated_config& c = b->cfg;
    const Named list[] = {{"x", &t.x, rows, c.p, false},           {"gate", &t.gate, c.p, c.hidden, false}, {"up", &t.up, c.p, c.hidden, false},
                          {"down", &t.down, c.hidden, c.out_n, false}, {"y", &t.y, rows, c.out_n, false},   {"g", &t.g, rows, c.hidden, true},
                          {"u", &t.u, rows, c.hidden, true}};
    GATED_DO(check(b, "bmgd_gated_forward", list, 7));
    if (!t.g.data != !t.u.data) return fail(b, BMGD_EINVAL, "bmgd_gated_forward", "g and u are kept together or not at all");
    if (rows == 0) return BMGD_OK;
    const OnDevice on(b->device);
    if (on.e != hipSuccess) return hip_fail(b, on.e, "hipSetDevice");
    GATED_DO(enter(b, s));
    const int64_t half = up(c.hidden, 64);
    GatedProduct q{}, y{};
    q.pair = y.pair = rows <= kGatedPairRows;
    const int64_t between = q.pair ? 2 * rows : rows;          // rows of H
    q.M = rows; q.N = c.hidden; q.K = c.p;
    q.half = half;
    plan(b, q, kOpUp, rows);
    y.M = between; y.N = c.out_n; y.K = c.hidden;
    plan(b, y, kOpMul, rows);

    Operands o{b};
    bool any, any_y;
    choose({b->wide && gated_can_be_loose(q.tile), unless(direct(t.x, rows, c.p), rows * c.p) + unless(pair_direct(t.gate, t.up, c.p, c.hidden), 2 * c.p * c.hidden), q.us},
           {b->wide && gated_can_be_loose(y.tile), unless(direct(t.down, c.hidden, c.out_n), c.hidden * c.out_n), y.us}, &any, &any_y);
    q.a = o.use(t.x, rows, c.p, b->lay.x, any, &q.loose);
    o.use_pair(t.gate, t.up, c.p, c.hidden, b->lay.gate, b->lay.up, any, &q.loose, &q.b, &q.b2);
    y.b = o.use(t.down, c.hidden, c.out_n, b->lay.down, any_y, &y.loose);
    if (o.pack.count) GATED_TRY(b, gated_launch_pack(o.pack, s));
    q.b_cols = q.loose ? c.hidden : up(c.hidden, 8);
    q.out = GatedMat{b->base + b->lay.h, half};
    q.g = plain(t.g);
    q.u = plain(t.u);
    b->turn ^= 1;
    scales(b, q, b->lay.scale_h);
    GATED_DO(launch(b, q, kOpUp, s));

    y.a = q.out;
    scales(b, y, b->lay.scale_h);
    y.b_cols = y.loose ? c.out_n : up(c.out_n, 8);
    y.out = plain(t.y);
    return launch(b, y, kOpMul, s);
}

int backward(bmgd_gated* b, int64_t rows, const bmgd_gated_tensors& t, hipStream_t s)
{
    const bmgd_gated_config& c = b->cfg;
    const Named list[] = {{"dy", &t.dy, rows, c.out_n, false},  {"x", &t.x, rows, c.p, false},          {"gate", &t.gate, c.p, c.hidden, false},
                          {"up", &t.up, c.p, c.hidden, false},  {"down", &t.down, c.hidden, c.out_n, false}, {"g", &t.g, rows, c.hidden, false},
                          {"u", &t.u, rows, c.hidden, false},   {"dx", &t.dx, rows, c.p, true},         {"dgate", &t.dgate, c.p, c.hidden, true},
                          {"dup", &t.dup, c.p, c.hidden, true}, {"ddown", &t.ddown, c.hidden, c.out_n, true}};
    GATED_DO(check(b, "bmgd_gated_backward", list, 11));
    if (!t.dgate.data != !t.dup.data) return fail(b, BMGD_EINVAL, "bmgd_gated_backward", "dgate and dup are wanted together or not at all");
    const OnDevice on(b->device);
    if (on.e != hipSuccess) return hip_fail(b, on.e, "hipSetDevice");
    GATED_DO(enter(b, s));
    const int64_t half = up(c.hidden, 64);
    const GatedMat h{b->base + b->lay.h, half}, d{b->base + b->lay.d, 2 * half};
    GatedProduct q{}, input{}, ddown{}, dgate{};
    q.pair = input.pair = ddown.twice_b = dgate.twice_a = rows <= kGatedPairRows;
    const int64_t between = q.pair ? 2 * rows : rows;          // rows of H and D
    GatedProduct* list3[3];
    GatedOp ops[3];
    int n = 0;
    if (rows) {
        q.M = rows; q.N = c.hidden; q.K = c.out_n;
        q.half = half;
        plan(b, q, kOpDown, rows);
    }
    if (rows && t.dx.data) {
        input.M = between; input.N = c.p; input.K = c.hidden;
        input.half = half;
        list3[n] = &input;
        ops[n++] = kOpInput;
    }
    if (t.ddown.data) {
        ddown.M = c.hidden; ddown.N = c.out_n; ddown.K = between;
        list3[n] = &ddown;
        ops[n++] = kOpWeight;
    }
    if (t.dgate.data) {
        dgate.M = c.p; dgate.N = c.hidden; dgate.K = between;
        dgate.half = half;
        list3[n] = &dgate;
        ops[n++] = kOpWeight;
    }
    if (n) plan(b, list3, ops, n, rows, 8 | (input.M ? 1 : 0) | (ddown.M ? 2 : 0) | (dgate.M ? 4 : 0));

    // (dY is read by both launches: where one needs a copy, both read that)
    Operands o{b};
    bool any, any_grads;
    const int64_t of_dy = unless(!rows || direct(t.dy, rows, c.out_n), rows * c.out_n);
    choose({b->wide && gated_can_be_loose(q.tile), of_dy + unless(direct(t.down, c.hidden, c.out_n), c.hidden * c.out_n), q.us},
           {b->wide && n && gated_can_be_loose(list3[0]->tile), unless(!ddown.M, of_dy) + unless(!rows || !dgate.M || direct(t.x, rows, c.p), rows * c.p) +
                unless(!input.M || pair_direct(t.gate, t.up, c.p, c.hidden), 2 * c.p * c.hidden), n ? list3[0]->us : 0.0}, &any, &any_grads);
    bool loose = false;
    const GatedMat dy = o.use(t.dy, rows, c.out_n, b->lay.dy, any && (any_grads || !ddown.M), &q.loose);
    if (ddown.M) loose = q.loose;
    q.b = o.use(t.down, c.hidden, c.out_n, b->lay.down, any, &q.loose);
    GatedMat x{};
    if (dgate.M) x = o.use(t.x, rows, c.p, b->lay.x, any_grads, &loose);
    if (input.M) o.use_pair(t.gate, t.up, c.p, c.hidden, b->lay.gate, b->lay.up, any_grads, &loose, &input.b, &input.b2);
    if (rows && o.pack.count) GATED_TRY(b, gated_launch_pack(o.pack, s));
    b->turn ^= 1;
    if (rows) {
        if (!q.loose) q.K = up(c.out_n, 8);
        scales(b, q, b->lay.scale_h, b->lay.scale_d);
        q.a = dy;
        q.out = h;
        q.out2 = d;
        q.g = plain(t.g);
        q.u = plain(t.u);
        GATED_DO(launch(b, q, kOpDown, s));
    }
    if (n == 0) return BMGD_OK;
    auto cols = [&](int64_t n) { return loose ? n : up(n, 8); };
    input.loose = ddown.loose = dgate.loose = loose;
    input.a = d;
    input.K = cols(c.hidden);
    input.out = plain(t.dx);
    ddown.a = h;
    ddown.b = dy;
    ddown.a_cols = half;
    ddown.b_cols = cols(c.out_n);
    ddown.out = plain(t.ddown);
    dgate.a = x;
    dgate.b = d;
    dgate.a_cols = cols(c.p);
    dgate.b_cols = 2 * half;
    dgate.out = plain(t.dgate);
    dgate.out2 = plain(t.dup);
    scales(b, input, b->lay.scale_d);
    scales(b, ddown, b->lay.scale_h);
    scales(b, dgate, b->lay.scale_d);
    const GatedProduct *pi = input.M ? &input : nullptr, *pd = ddown.M ? &ddown : nullptr, *pg = dgate.M ? &dgate : nullptr;
    const hipError_t e = c.dtype == BMGD_F16 ? gated_launch_grads_f16(pi, pd, pg, s) : gated_launch_grads_bf16(pi, pd, pg, s);
    if (e != hipSuccess) return hip_fail(b, e, "launch of the gradients of the gated block");
    return BMGD_OK;
}

// The kernels' shared memory, once per device and type.
hipError_t prepare_once(int device, bool f16)
{
    constexpr int kDevices = 64;
    static std::atomic<bool> done[kDevices][2];
    const bool known = device >= 0 && device < kDevices;
    if (known && done[device][f16].load(std::memory_order_acquire)) return hipSuccess;
    const hipError_t e = f16 ? gated_prepare_f16() : gated_prepare_bf16();
    if (e == hipSuccess && known) done[device][f16].store(true, std::memory_order_release);
    return e;
}

void destroy(bmgd_gated* b)
{
    if (!b) return;
    int current = -1;
    (void)hipGetDevice(&current);
    if (hipSetDevice(b->device) == hipSuccess) {
        if (b->used || b->captured) (void)hipDeviceSynchronize();
        if (b->order) (void)hipEventDestroy(b->order);
        if (b->owned && b->base) (void)hipFree(b->base);
    }
    if (current >= 0) (void)hipSetDevice(current);
    (void)hipGetLastError();
    delete b;
}

}  // namespace

#define BMGD_API __attribute__((visibility("default")))

extern "C" {

BMGD_API size_t bmgd_gated_workspace_bytes(const bmgd_gated_config* cfg)
{
    const char* why = "";
    return cfg && valid(*cfg, &why) ? make_layout(*cfg).total : 0;
}

BMGD_API int bmgd_gated_create(const bmgd_gated_config* cfg, bmgd_gated** out)
{
    if (out) *out = nullptr;
    if (!cfg || !out) return fail_static(BMGD_EINVAL, "bmgd_gated_create", "cfg and out must not be NULL");
    const char* why = "";
    if (!valid(*cfg, &why)) return fail_static(BMGD_EINVAL, "bmgd_gated_create", why);
    const Layout lay = make_layout(*cfg);
    if (cfg->workspace && ((uintptr_t)cfg->workspace & 255)) return fail_static(BMGD_EINVAL, "bmgd_gated_create", "workspace must be 256-byte aligned");
    if (cfg->workspace && cfg->workspace_bytes < lay.total) return fail_static(BMGD_ENOMEM, "bmgd_gated_create", "workspace too small");
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || ndev == 0) {
        (void)hipGetLastError();
        return fail_static(BMGD_EHIP, "bmgd_gated_create", "no HIP device available");
    }
    bmgd_gated* b = new (std::nothrow) bmgd_gated();
    if (!b) return fail_static(BMGD_ENOMEM, "bmgd_gated_create", "out of host memory");
    b->cfg = *cfg;
    b->lay = lay;
    b->wide = std::min(std::min(cfg->p, cfg->hidden), cfg->out_n) >= 8;
    auto bail = [&](hipError_t e, const char* what) {
        const int code = hip_fail(b, e, what);
        set_create_error(b->err);
        destroy(b);
        return code;
    };
    hipError_t e = hipGetDevice(&b->device);
    if (e != hipSuccess) return bail(e, "hipGetDevice");
    e = hipDeviceGetAttribute(&b->num_cus, hipDeviceAttributeMultiprocessorCount, b->device);
    if (e != hipSuccess) return bail(e, "hipDeviceGetAttribute");
    e = prepare_once(b->device, cfg->dtype == BMGD_F16);
    if (e != hipSuccess) return bail(e, "hipFuncSetAttribute");
    e = hipEventCreateWithFlags(&b->order, hipEventDisableTiming);
    if (e != hipSuccess) return bail(e, "hipEventCreateWithFlags");
    if (cfg->workspace) {
        b->base = static_cast<char*>(cfg->workspace);
    } else {
        void* p = nullptr;
        e = hipMalloc(&p, lay.total);
        if (e != hipSuccess) return bail(e, "hipMalloc");
        b->base = static_cast<char*>(p);
        b->owned = true;
    }
    e = launch_fill_zero(b->base + lay.counter, lay.total - lay.counter, nullptr);
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
    if (e != hipSuccess) return bail(e, "clearing the workspace");
    *out = b;
    return BMGD_OK;
}

BMGD_API int bmgd_gated_forward(bmgd_gated* block, int64_t rows, const bmgd_gated_tensors* t, void* stream)
{
    if (!block) return fail_static(BMGD_EINVAL, "bmgd_gated_forward", "block must not be NULL");
    if (!t) return fail(block, BMGD_EINVAL, "bmgd_gated_forward", "tensors must not be NULL");
    if (rows < 0 || rows > block->cfg.max_rows) return fail(block, BMGD_EINVAL, "bmgd_gated_forward", "rows must be in [0, max_rows]");
    return forward(block, rows, *t, static_cast<hipStream_t>(stream));
}

BMGD_API int bmgd_gated_backward(bmgd_gated* block, int64_t rows, const bmgd_gated_tensors* t, void* stream)
{
    if (!block) return fail_static(BMGD_EINVAL, "bmgd_gated_backward", "block must not be NULL");
    if (!t) return fail(block, BMGD_EINVAL, "bmgd_gated_backward", "tensors must not be NULL");
    if (rows < 0 || rows > block->cfg.max_rows) return fail(block, BMGD_EINVAL, "bmgd_gated_backward", "rows must be in [0, max_rows]");
    return backward(block, rows, *t, static_cast<hipStream_t>(stream));
}

BMGD_API const char* bmgd_gated_last_error(const bmgd_gated* block)
{
    return block ? block->err : bmgd_last_error(nullptr);
}

BMGD_API void bmgd_gated_destroy(bmgd_gated* block) { destroy(block); }

// For tests: the kind of tile and the shares of a tile's sum that later calls use where they fit; tile < 0: their own choice again.
BMGD_API int bmgd_internal_gated_tile(bmgd_gated* block, int32_t tile, int32_t shares)
{
    if (!block || tile >= kTiles || shares < 1 || shares > 64) return BMGD_EINVAL;
    block->tile = tile;
    block->shares = shares;
    return BMGD_OK;
}

}  // extern "C"
