// C-ABI entry points of the operators around the attention: argument validation, then the launches.
// Tensors here have strides; what a call may overlap is decided from them before anything is enqueued.
#include <limits.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <initializer_list>

#include "../../include/sfda.h"
#include "sfda_layer.h"

namespace {

typedef long long ll;

bool dtype_ok(sfda_dtype_t d) { return d == SFDA_F32 || d == SFDA_BF16; }
ll esize(sfda_dtype_t d) { return d == SFDA_BF16 ? 2 : 4; }

// a tensor: up to three outer axes and D contiguous elements; strides and offsets in bytes
struct Box {
    const void* p;
    ll n[4], s[4];
    int axes;
};

constexpr ll FAR = 1LL << 46;       // past any device memory: strides and sizes are kept below it

Box box(const void* p, ll e, ll D, std::initializer_list<ll> n, const ll* strides)
{
    Box b{p, {}, {}, 0};
    int i = 0;
    for (ll m : n) {
        b.n[i] = m;
        b.s[i] = strides[i] < 0 || strides[i] > FAR ? -1 : strides[i] * e;      // (-1: refused by extent)
        ++i;
    }
    b.n[i] = D * e;
    b.s[i] = 1;
    b.axes = i + 1;
    return b;
}

bool empty(const Box& b)
{
    for (int i = 0; i < b.axes; ++i)
        if (b.n[i] == 0) return true;
    return false;
}

// bytes from the first element's to past the last element's; -1 where a stride is negative or the sum is out of range
ll extent(const Box& b)
{
    ll last = 0;
    for (int i = 0; i < b.axes; ++i) {
        if (b.s[i] < 0 || b.s[i] > FAR || b.n[i] > FAR) return -1;
        if (b.n[i] > 1) {
            if (b.s[i] != 0 && b.n[i] - 1 > FAR / b.s[i]) return -1;
            last += (b.n[i] - 1) * b.s[i];
        }
        if (last > FAR) return -1;
    }
    return last + 1;
}

// the axes by falling stride; nested: every axis steps past all that the smaller ones span, so that no
// two elements share a place
struct Order {
    int axis[4];
    bool nested;
};
Order order(const Box& b)
{
    Order o{{0, 1, 2, 3}, true};
    std::sort(o.axis, o.axis + b.axes, [&](int x, int y) { return b.s[x] > b.s[y]; });
    ll span = 0;
    for (int i = b.axes - 1; i >= 0; --i) {
        const int a = o.axis[i];
        if (b.n[a] <= 1) continue;
        if (b.s[a] <= span) o.nested = false;
        span += (b.n[a] - 1) * b.s[a];
    }
    return o;
}

// whether some i with -(y.n - 1) <= i <= x.n - 1 on each axis has sum i s = delta, s the strides of x
bool meets(const Box& x, const Box& y, const Order& o, int at, ll delta)
{
    if (at == x.axes) return delta == 0;
    const int a = o.axis[at];
    const ll s = x.s[a];
    if (s == 0) return meets(x, y, o, at + 1, delta);
    const ll low = delta >= 0 ? delta / s : -((-delta + s - 1) / s);
    for (ll i = low; i <= low + 1; ++i)
        if (i >= -(y.n[a] - 1) && i <= x.n[a] - 1 && meets(x, y, o, at + 1, delta - i * s)) return true;
    return false;
}

// Whether two tensors share a byte.  Slices of one buffer (the same strides) are told apart exactly,
// other tensors by the ranges they lie in.
bool overlap(const Box& x, const Box& y)
{
    if (x.p == nullptr || y.p == nullptr || empty(x) || empty(y)) return false;
    const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
    if (a + static_cast<uintptr_t>(extent(x)) <= b || b + static_cast<uintptr_t>(extent(y)) <= a) return false;
    if (x.axes != y.axes) return true;
    // each axis as long as the longer one; of an axis of one element the other tensor's stride counts, or none
    Box all = x, u = x;
    for (int i = 0; i < x.axes; ++i) {
        if (x.n[i] > 1 && y.n[i] > 1 && x.s[i] != y.s[i]) return true;
        all.n[i] = std::max(x.n[i], y.n[i]);
        all.s[i] = u.s[i] = x.n[i] > 1 ? x.s[i] : y.n[i] > 1 ? y.s[i] : 0;
    }
    const Order o = order(all);
    if (!o.nested) return true;
    return meets(u, y, o, 0, b > a ? static_cast<ll>(b - a) : -static_cast<ll>(a - b));
}

bool same(const Box& x, const Box& y)
{
    if (x.p != y.p) return false;
    for (int i = 0; i < x.axes; ++i)
        if (x.n[i] > 1 && x.s[i] != y.s[i]) return false;
    return true;
}

Box flat(const void* p, ll bytes)
{
    const ll s[1] = {0};
    return box(p, 1, bytes, {1}, s);
}

// Pointers, strides and overlaps of a call: `need` pointers are not NULL, every one is aligned to its
// elements, no output meets an input (but for the pairs in place) or another output.
struct Call {
    static constexpr int MAX = 20;
    Box in[MAX], out[MAX];
    ll in_place[MAX];       // index of the input that an output may equal, -1 none
    int ins = 0, outs = 0;
    sfda_status_t st = SFDA_OK;

    void fail(sfda_status_t s) { if (st == SFDA_OK) st = s; }
    void check(const Box& b, ll align, bool need)
    {
        if (b.p == nullptr) {
            if (need && !empty(b)) fail(SFDA_ERR_NULL);
            return;
        }
        if (extent(b) < 0) fail(SFDA_ERR_SHAPE);
        if (reinterpret_cast<uintptr_t>(b.p) % static_cast<uintptr_t>(align) != 0) fail(SFDA_ERR_ALIGN);
    }
    int input(const Box& b, ll align, bool need = true)
    {
        check(b, align, need);
        in[ins] = b;
        return ins++;
    }
    void output(const Box& b, ll align, bool need = true, ll place = -1)
    {
        check(b, align, need);
        out[outs] = b;
        in_place[outs++] = place;
    }
    sfda_status_t done() const
    {
        if (st != SFDA_OK) return st;
        for (int i = 0; i < outs; ++i) {
            if (out[i].p == nullptr || empty(out[i])) continue;
            if (!order(out[i]).nested) return SFDA_ERR_ALIAS;
            for (int j = 0; j < ins; ++j)
                if (!(in_place[i] == j && same(out[i], in[j])) && overlap(out[i], in[j])) return SFDA_ERR_ALIAS;
            for (int j = 0; j < i; ++j)
                if (overlap(out[i], out[j])) return SFDA_ERR_ALIAS;
        }
        return SFDA_OK;
    }
};

// The strides of a tensor's outer axes: the caller's, or a contiguous tensor's.  Those of axes of one element, which a caller may
// give any value, are 0 from here on: the scan reaches its blocks' rows by whole blocks, and a token that is alone lies in one.
template <int N> void strides_of(ll (&out)[N], const ll* given, const ll (&n)[N], const ll (&contiguous)[N])
{
    for (int i = 0; i < N; ++i) out[i] = n[i] <= 1 ? 0 : given != nullptr ? given[i] : contiguous[i];
}
// [B, H, T, D], the `which`-th of a call
void strides3(ll (&out)[3], const ll* given, int which, ll B, ll H, ll T, ll D)
{
    strides_of(out, given != nullptr ? given + 3 * which : nullptr, {B, H, T}, {H * T * D, T * D, D});
}

// compute units of the current device, looked up once for each
int cus()
{
    static std::atomic<int> known[64];
    int dev = -1, v = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    if ((v = known[dev].load(std::memory_order_relaxed)) > 0) return v;
    if (hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v <= 0) return 256;
    known[dev].store(v, std::memory_order_relaxed);
    return v;
}

constexpr int MAX_D = 256;              // key and value channels of a decay attention
bool decay_sizes(int B, int H, int T, int dk, int dv)
{
    if (B < 0 || H < 0 || T < 0 || dk < 1 || dk > MAX_D || dv < 1 || dv > MAX_D) return false;
    // at most 8 threads for a head and value column of a role, in launches of less than 2^32 (by a division: B H alone may have 62
    // bits); tokens are counted in 32 bits with room for a block
    return static_cast<ll>(B) * H <= ((1LL << 32) - 1) / (3 * MAX_D * 8) && T <= INT_MAX - 1024;
}

// a block's rows (at most 64 tokens) are addressed with 32-bit byte offsets
bool rows_fit(const ll (&st)[3], ll e) { return st[2] <= ((1LL << 31) - 65536) / (64 * e); }

// Segments of a sequence.  A scan without them takes c us for 64 tokens, whatever the number of heads, until the workgroups fill the
// compute units.  Cut into S parts it takes a pass for their states (another s c us) and a join, all of them on an S-th of the
// tokens, with one workgroup on each unit, or with two of bfloat16.  The estimates are in us, for the padded channels of the state
// and for rows of whole vectors or not; roles of different padding add up, but where they share a launch.
// Measured, whole / cut, us of a call among others, d 128: bfloat16 forward 16 heads T 512 23/27, 4 heads T 256 17/24, 15 heads T 1003
// 39/36 (keys of 88, values of 74: 54/33), 32 heads T 2048 72/48; backward 16 heads T 512 25/37, 32 heads T 2048 72/90; float32
// forward 4 heads T 512 56/29, 32 heads T 2048 199/98; backward 16 heads T 512 60/61, 32 heads T 2048 201/194; d 64, 16 heads T 2048
// 125/34; d 256, 4 heads T 512 81/38.
struct Cut { int tokens, segments; };
struct State { int da, db; };           // a role's
Cut cut_of(ll heads, std::initializer_list<State> roles, int T, bool bf16)
{
    int widest = 0;
    bool vectors = true;
    ll groups[3] = {0, 0, 0}, together = 0;
    auto padded = [](int da) { return da <= 64 ? 0 : da <= 128 ? 1 : 2; };
    for (const State& r : roles) {
        widest = std::max(widest, padded(r.da));
        groups[padded(r.da)] += heads * sfda::decay_slices(bf16, r.da, r.db);
        vectors = vectors && (r.da | r.db) % (bf16 ? 8 : 4) == 0;
    }
    for (const State& r : roles) together += heads * sfda::decay_slices(bf16, 64 << widest, r.db);
    auto cost = [&](ll segments) {
        constexpr double B[3] = {2.4, 2.4, 4.8}, F[3] = {3.7, 6.2, 9.3};
        double c = 0;
        for (int i = 0; i < 3; ++i)
            if (together * segments <= cus() ? i == widest : groups[i] > 0) c += bf16 ? B[i] : F[i];
        return vectors ? c : 1.5 * c;
    };
    const double s = bf16 ? 0.6 : 0.5, shared = 1.6;        // the states' pass to the other; two on a unit: each slower
    const ll steps = (static_cast<ll>(T) + 63) / 64;
    Cut best{std::max(T, 1), 1};
    double least = 0.9 * (steps * cost(1) + 5.);
    for (int on_unit = 1; on_unit <= (bf16 ? 2 : 1); ++on_unit) {
        const ll most = on_unit * static_cast<ll>(cus()) / std::max({groups[0], groups[1], groups[2]});
        if (most < 2 || steps < 2) continue;
        const ll each = (steps + most - 1) / most, segments = (steps + each - 1) / each;        // steps of a segment
        const double us = each * cost(segments) * (1 + s) * (on_unit == 2 ? shared : 1.) + 20.;
        if (us < least) {
            least = us;
            best = {static_cast<int>(each * 64), static_cast<int>(segments)};
        }
    }
    return best;
}
// dq and dk have dk columns, dv has dv
Cut cut_fwd(ll heads, int T, int dk, int dv, bool bf16) { return cut_of(heads, {{dk, dv}}, T, bf16); }
Cut cut_bwd(ll heads, int T, int dk, int dv, bool bf16) { return cut_of(heads, {{dv, dk}, {dv, dk}, {dk, dv}}, T, bf16); }

}  // namespace

extern "C" {

sfda_status_t sfda_rotary(const void* q, const void* k, const float* cos, const float* sin, const void* positions,
                          int position_bits, long long position_stride, long long offset, void* qo, void* ko, int B,
                          int Hq, int Hk, int T, int D, int rot, int P, int interleaved, int inverse,
                          const long long* strides, sfda_dtype_t dtype, sfda_stream_t stream)
{
    if (!dtype_ok(dtype)) return SFDA_ERR_DTYPE;
    if (B < 0 || Hq < 0 || Hk < 0 || T < 0 || D < 1 || D > 4096 || rot < 2 || rot > D || (rot & 1) || P < 1) return SFDA_ERR_SHAPE;
    if (positions != nullptr && ((position_bits != 32 && position_bits != 64) || position_stride < 0)) return SFDA_ERR_SHAPE;
    if (positions == nullptr && T > 0 && (offset < 0 || offset > P - static_cast<ll>(T))) return SFDA_ERR_SHAPE;
    if (k == nullptr) Hk = 0;
    if (static_cast<ll>(Hq) + Hk > INT_MAX - 64) return SFDA_ERR_SHAPE;
    if (B == 0 || T == 0 || Hq + Hk == 0) return SFDA_OK;
    const ll e = esize(dtype);
    // a thread for four heads or four tokens of a 16-byte unit of channels, less than 2^32 in a launch
    const double H = static_cast<double>(Hq) + Hk, rows = std::max((H + 6) / 4 * T, H * ((T + 3.) / 4)) * B;
    if (rows * (D * e / 16. + 3) >= 4294967296. - 1024.) return SFDA_ERR_SHAPE;
    sfda::RotaryLaunch L{};
    strides3(L.q_s, strides, 0, B, Hq, T, D);
    strides3(L.k_s, strides, 1, B, Hk, T, D);
    strides3(L.qo_s, strides, 2, B, Hq, T, D);
    strides3(L.ko_s, strides, 3, B, Hk, T, D);
    Call c;
    const int iq = c.input(box(q, e, D, {B, Hq, T}, L.q_s), e);
    const int ik = c.input(box(k, e, D, {B, Hk, T}, L.k_s), e);
    c.input(flat(cos, static_cast<ll>(P) * (rot / 2) * 4), 4);
    c.input(flat(sin, static_cast<ll>(P) * (rot / 2) * 4), 4);
    if (positions != nullptr) {
        const ll ps[1] = {position_stride};
        c.input(box(positions, position_bits / 8, T, {B}, ps), position_bits / 8);
    }
    c.output(box(qo, e, D, {B, Hq, T}, L.qo_s), e, true, iq);
    c.output(box(ko, e, D, {B, Hk, T}, L.ko_s), e, true, ik);
    const sfda_status_t st = c.done();
    if (st != SFDA_OK) return st;
    L.q = q; L.k = k; L.qo = qo; L.ko = ko; L.cos = cos; L.sin = sin;
    L.positions = positions; L.pos64 = position_bits == 64; L.pos_b = position_stride; L.offset = offset;
    L.B = B; L.Hq = Hq; L.Hk = Hk; L.T = T; L.D = D; L.rot = rot; L.P = P;
    L.interleaved = interleaved != 0; L.inverse = inverse != 0; L.bf16 = dtype == SFDA_BF16;
    return sfda::launch_rotary(L, static_cast<hipStream_t>(stream)) == hipSuccess ? SFDA_OK : SFDA_ERR_HIP;
}

size_t sfda_decay_attn_fwd_workspace_bytes(int B, int H, int T, int dk, int dv, sfda_dtype_t dtype)
{
    if (!dtype_ok(dtype) || !decay_sizes(B, H, T, dk, dv)) return 0;
    const ll heads = static_cast<ll>(B) * H;
    const bool bf16 = dtype == SFDA_BF16;
    if (heads == 0) return 0;
    const Cut c = cut_fwd(heads, T, dk, dv, bf16);
    return c.segments > 1 ? static_cast<size_t>(c.segments) * heads * dk * dv * 4 : 0;
}

sfda_status_t sfda_decay_attn_fwd(const void* q, const void* k, const void* v, const float* log_decay, const int* lengths,
                                  const float* S0, void* o, float* S_T, int B, int H, int T, int dk, int dv, float scale,
                                  const long long* strides, sfda_dtype_t dtype, void* workspace, size_t workspace_bytes,
                                  sfda_stream_t stream)
{
    if (!dtype_ok(dtype)) return SFDA_ERR_DTYPE;
    if (!decay_sizes(B, H, T, dk, dv)) return SFDA_ERR_SHAPE;
    const ll heads = static_cast<ll>(B) * H, e = esize(dtype), state = heads * dk * dv * 4;
    const bool bf16 = dtype == SFDA_BF16;
    if (heads == 0) return SFDA_OK;
    sfda::DecayLaunch L{};
    sfda::DecayRole& R = L.role[0];
    strides3(R.q_s, strides, 0, B, H, T, dk);
    strides3(R.k_s, strides, 1, B, H, T, dk);
    strides3(R.v_s, strides, 2, B, H, T, dv);
    strides3(R.o_s, strides, 3, B, H, T, dv);
    if (!rows_fit(R.q_s, e) || !rows_fit(R.k_s, e) || !rows_fit(R.v_s, e) || !rows_fit(R.o_s, e)) return SFDA_ERR_SHAPE;
    const size_t need = sfda_decay_attn_fwd_workspace_bytes(B, H, T, dk, dv, dtype);
    const bool cut = need > 0 && workspace != nullptr && workspace_bytes >= need;
    Call c;
    c.input(box(q, e, dk, {B, H, T}, R.q_s), e);
    c.input(box(k, e, dk, {B, H, T}, R.k_s), e);
    c.input(box(v, e, dv, {B, H, T}, R.v_s), e);
    c.input(flat(log_decay, 4LL * H), 4);
    c.input(flat(lengths, 4LL * B), 4, false);
    const int s0 = c.input(flat(S0, state), 4, false);
    c.output(box(o, e, dv, {B, H, T}, R.o_s), e);
    c.output(flat(S_T, state), 4, false, s0);
    c.output(flat(cut ? workspace : nullptr, static_cast<ll>(need)), 4, false);
    const sfda_status_t st = c.done();
    if (st != SFDA_OK) return st;
    const Cut segs = cut_fwd(heads, T, dk, dv, bf16);
    R.q = q; R.k = k; R.v = v; R.o = o; R.S0 = S0; R.S_T = S_T;
    R.da = dk; R.db = dv; R.s_row = dv; R.s_col = 1;
    R.intra = scale; R.inter = scale; R.upd = 1.f;
    R.ws = cut ? static_cast<float*>(workspace) : nullptr;
    L.roles = 1; L.log_decay = log_decay; L.lengths = lengths; L.B = B; L.H = H; L.T = T;
    L.seg_tokens = cut ? segs.tokens : std::max(T, 1);
    L.segments = cut ? segs.segments : 1;
    L.cus = cus();
    L.bf16 = bf16;
    return sfda::launch_decay(L, static_cast<hipStream_t>(stream)) == hipSuccess ? SFDA_OK : SFDA_ERR_HIP;
}

// the dk and dv scans need dS_T, the dq scan S0
size_t sfda_decay_attn_bwd_workspace_bytes(int B, int H, int T, int dk, int dv, sfda_dtype_t dtype)
{
    if (!dtype_ok(dtype) || !decay_sizes(B, H, T, dk, dv)) return 0;
    const ll heads = static_cast<ll>(B) * H;
    const bool bf16 = dtype == SFDA_BF16;
    if (heads == 0) return 0;
    const Cut c = cut_bwd(heads, T, dk, dv, bf16);
    return c.segments > 1 ? 3 * static_cast<size_t>(c.segments) * heads * dk * dv * 4 : 0;
}

sfda_status_t sfda_decay_attn_bwd(const void* q, const void* k, const void* v, const float* log_decay, const int* lengths,
                                  const float* S0, const void* dO, const float* dS_T, void* dq, void* dk_out, void* dv_out,
                                  float* dS0, int B, int H, int T, int dk, int dv, float scale, const long long* strides,
                                  sfda_dtype_t dtype, void* workspace, size_t workspace_bytes, sfda_stream_t stream)
{
    if (!dtype_ok(dtype)) return SFDA_ERR_DTYPE;
    if (!decay_sizes(B, H, T, dk, dv)) return SFDA_ERR_SHAPE;
    const ll heads = static_cast<ll>(B) * H, e = esize(dtype), state = heads * dk * dv * 4;
    const bool bf16 = dtype == SFDA_BF16;
    if (heads == 0) return SFDA_OK;
    ll qs[3], ks[3], vs[3], gs[3], dqs[3], dks[3], dvs[3];
    strides3(qs, strides, 0, B, H, T, dk);
    strides3(ks, strides, 1, B, H, T, dk);
    strides3(vs, strides, 2, B, H, T, dv);
    strides3(gs, strides, 3, B, H, T, dv);
    strides3(dqs, strides, 4, B, H, T, dk);
    strides3(dks, strides, 5, B, H, T, dk);
    strides3(dvs, strides, 6, B, H, T, dv);
    for (const auto* st : {&qs, &ks, &vs, &gs, &dqs, &dks, &dvs})
        if (!rows_fit(*st, e)) return SFDA_ERR_SHAPE;
    const size_t need = sfda_decay_attn_bwd_workspace_bytes(B, H, T, dk, dv, dtype);
    const bool cut = need > 0 && workspace != nullptr && workspace_bytes >= need;
    Call c;
    c.input(box(q, e, dk, {B, H, T}, qs), e);
    c.input(box(k, e, dk, {B, H, T}, ks), e);
    c.input(box(v, e, dv, {B, H, T}, vs), e);
    c.input(box(dO, e, dv, {B, H, T}, gs), e);
    c.input(flat(log_decay, 4LL * H), 4);
    c.input(flat(lengths, 4LL * B), 4, false);
    c.input(flat(S0, state), 4, false);
    c.input(flat(dS_T, state), 4, false);
    c.output(box(dq, e, dk, {B, H, T}, dqs), e);
    c.output(box(dk_out, e, dk, {B, H, T}, dks), e);
    c.output(box(dv_out, e, dv, {B, H, T}, dvs), e);
    c.output(flat(dS0, state), 4, false);
    c.output(flat(cut ? workspace : nullptr, static_cast<ll>(need)), 4, false);
    const sfda_status_t st = c.done();
    if (st != SFDA_OK) return st;
    const Cut segs = cut_bwd(heads, T, dk, dv, bf16);
    const int segments = cut ? segs.segments : 1;
    sfda::DecayLaunch L{};
    auto put = [](ll (&to)[3], const ll (&from)[3]) { std::copy(from, from + 3, to); };
    auto role = [&](int i, const void* a, const ll (&as)[3], const void* b, const ll (&bs)[3], const void* x, const ll (&xs)[3], void* out,
                    const ll (&os)[3], int da, int db, bool transposed, bool reverse) {
        sfda::DecayRole& R = L.role[i];
        R.q = a; R.k = b; R.v = x; R.o = out;
        put(R.q_s, as); put(R.k_s, bs); put(R.v_s, xs); put(R.o_s, os);
        R.da = da; R.db = db;
        R.s_row = transposed ? 1 : dv; R.s_col = transposed ? dv : 1;
        R.S0 = reverse ? dS_T : S0; R.S_T = nullptr; R.reverse = reverse;
        R.intra = scale; R.inter = reverse ? 1.f : scale; R.upd = reverse ? scale : 1.f;
        R.ws = cut ? static_cast<float*>(workspace) + i * static_cast<ll>(segments) * heads * dk * dv : nullptr;
    };
    role(0, v, vs, dO, gs, q, qs, dk_out, dks, dv, dk, true, true);
    role(1, k, ks, q, qs, dO, gs, dv_out, dvs, dk, dv, false, true);
    role(2, dO, gs, v, vs, k, ks, dq, dqs, dv, dk, true, false);
    L.role[1].S_T = dS0;
    L.roles = 3; L.log_decay = log_decay; L.lengths = lengths; L.B = B; L.H = H; L.T = T;
    L.seg_tokens = cut ? segs.tokens : std::max(T, 1);
    L.segments = segments;
    L.cus = cus();
    L.bf16 = bf16;
    return sfda::launch_decay(L, static_cast<hipStream_t>(stream)) == hipSuccess ? SFDA_OK : SFDA_ERR_HIP;
}

sfda_status_t sfda_decay_attn_step(const void* q, const void* k, const void* v, const float* log_decay, float* S, void* o,
                                   int B, int H, int dk, int dv, float scale, const long long* strides, sfda_dtype_t dtype,
                                   sfda_stream_t stream)
{
    if (!dtype_ok(dtype)) return SFDA_ERR_DTYPE;
    if (!decay_sizes(B, H, 1, dk, dv)) return SFDA_ERR_SHAPE;
    const ll heads = static_cast<ll>(B) * H, e = esize(dtype);
    if (heads == 0) return SFDA_OK;
    sfda::DecayStepLaunch L{};
    ll (*to[4])[2] = {&L.q_s, &L.k_s, &L.v_s, &L.o_s};
    for (int i = 0; i < 4; ++i) {
        const ll D = i < 2 ? dk : dv;
        strides_of(*to[i], strides != nullptr ? strides + 2 * i : nullptr, {B, H}, {H * D, D});
    }
    Call c;
    c.input(box(q, e, dk, {B, H}, L.q_s), e);
    c.input(box(k, e, dk, {B, H}, L.k_s), e);
    c.input(box(v, e, dv, {B, H}, L.v_s), e);
    c.input(flat(log_decay, 4LL * H), 4);
    c.output(flat(S, heads * dk * dv * 4), 4);
    c.output(box(o, e, dv, {B, H}, L.o_s), e);
    const sfda_status_t st = c.done();
    if (st != SFDA_OK) return st;
    L.q = q; L.k = k; L.v = v; L.o = o; L.S = S; L.log_decay = log_decay;
    L.B = B; L.H = H; L.dk = dk; L.dv = dv; L.scale = scale; L.bf16 = dtype == SFDA_BF16;
    return sfda::launch_decay_step(L, static_cast<hipStream_t>(stream)) == hipSuccess ? SFDA_OK : SFDA_ERR_HIP;
}

static bool norm_sizes(int B, int H, int T, int D)
{
    return B >= 0 && H >= 0 && T >= 0 && D >= 1 && D <= sfda::NORM_MAX && static_cast<ll>(H) * D <= (1LL << 30) && H <= (1 << 23);
}

// strides [x: b, h, t][then pairs b, t], or contiguous ones
static void norm_strides(ll (&x)[3], const ll* given, ll B, ll H, ll T, ll D) { strides3(x, given, 0, B, H, T, D); }
static void pair_strides(ll (&out)[2], const ll* given, int at, ll B, ll H, ll T, ll D)
{
    strides_of(out, given != nullptr ? given + at : nullptr, {B, T}, {T * H * D, H * D});
}

sfda_status_t sfda_group_norm(const void* x, const float* weight, const float* bias, const void* gate, void* y, int B, int H,
                              int T, int D, int activation, float eps, const long long* strides, sfda_dtype_t dtype,
                              sfda_stream_t stream)
{
    if (!dtype_ok(dtype)) return SFDA_ERR_DTYPE;
    if (!norm_sizes(B, H, T, D) || (activation != SFDA_ACT_NONE && activation != SFDA_ACT_SILU) || !(eps >= 0.f)) return SFDA_ERR_SHAPE;
    if (B == 0 || H == 0 || T == 0) return SFDA_OK;
    const ll e = esize(dtype), HD = static_cast<ll>(H) * D;
    sfda::NormLaunch L{};
    norm_strides(L.x_s, strides, B, H, T, D);
    pair_strides(L.g_s, strides, 3, B, H, T, D);
    pair_strides(L.y_s, strides, 5, B, H, T, D);
    Call c;
    c.input(box(x, e, D, {B, H, T}, L.x_s), e);
    c.input(flat(weight, 4 * HD), 4, false);
    c.input(flat(bias, 4 * HD), 4, false);
    c.input(box(gate, e, HD, {B, T}, L.g_s), e, false);
    c.output(box(y, e, HD, {B, T}, L.y_s), e);
    const sfda_status_t st = c.done();
    if (st != SFDA_OK) return st;
    L.x = x; L.weight = weight; L.bias = bias; L.gate = gate; L.y = y;
    L.B = B; L.H = H; L.T = T; L.D = D; L.silu = activation == SFDA_ACT_SILU; L.eps = eps; L.bf16 = dtype == SFDA_BF16;
    return sfda::launch_norm(L, static_cast<hipStream_t>(stream)) == hipSuccess ? SFDA_OK : SFDA_ERR_HIP;
}

size_t sfda_group_norm_bwd_workspace_bytes(int B, int H, int T, int D, sfda_dtype_t dtype)
{
    if (!dtype_ok(dtype) || !norm_sizes(B, H, T, D) || H == 0) return 0;
    return static_cast<size_t>(sfda::norm_strips(static_cast<long>(B) * T, H, D, dtype == SFDA_BF16)) * 2 * H * D * 4;
}

sfda_status_t sfda_group_norm_bwd(const void* dy, const void* x, const float* weight, const float* bias, const void* gate,
                                  void* dx, void* dgate, float* dweight, float* dbias, int B, int H, int T, int D,
                                  int activation, float eps, const long long* strides, sfda_dtype_t dtype, void* workspace,
                                  size_t workspace_bytes, sfda_stream_t stream)
{
    if (!dtype_ok(dtype)) return SFDA_ERR_DTYPE;
    if (!norm_sizes(B, H, T, D) || (activation != SFDA_ACT_NONE && activation != SFDA_ACT_SILU) || !(eps >= 0.f)) return SFDA_ERR_SHAPE;
    if (H == 0) return SFDA_OK;
    const ll e = esize(dtype), HD = static_cast<ll>(H) * D;
    const size_t need = dweight != nullptr || dbias != nullptr ? sfda_group_norm_bwd_workspace_bytes(B, H, T, D, dtype) : 0;
    sfda::NormLaunch L{};
    norm_strides(L.x_s, strides, B, H, T, D);
    pair_strides(L.g_s, strides, 3, B, H, T, D);
    pair_strides(L.y_s, strides, 5, B, H, T, D);
    norm_strides(L.dx_s, strides != nullptr ? strides + 7 : nullptr, B, H, T, D);
    pair_strides(L.dg_s, strides, 10, B, H, T, D);
    Call c;
    c.input(box(dy, e, HD, {B, T}, L.y_s), e);
    c.input(box(x, e, D, {B, H, T}, L.x_s), e);
    c.input(flat(weight, 4 * HD), 4, false);
    c.input(flat(bias, 4 * HD), 4, false);
    c.input(box(gate, e, HD, {B, T}, L.g_s), e, false);
    c.output(box(dx, e, D, {B, H, T}, L.dx_s), e);
    c.output(box(dgate, e, HD, {B, T}, L.dg_s), e, gate != nullptr);
    c.output(flat(dweight, 4 * HD), 4, false);
    c.output(flat(dbias, 4 * HD), 4, false);
    if (need > 0) c.output(flat(workspace, static_cast<ll>(need)), 4);
    sfda_status_t st = c.done();
    if (st == SFDA_OK && need > 0 && workspace_bytes < need) st = SFDA_ERR_SHAPE;
    if (st != SFDA_OK) return st;
    L.dy = dy; L.x = x; L.weight = weight; L.bias = bias; L.gate = gate;
    L.dx = dx; L.dgate = dgate; L.dweight = dweight; L.dbias = dbias;
    L.partial = dweight != nullptr || dbias != nullptr ? static_cast<float*>(workspace) : nullptr;
    L.B = T > 0 ? B : 0; L.H = H; L.T = std::max(T, 1); L.D = D;      // (no tokens: the weights' gradients are zeros)
    L.silu = activation == SFDA_ACT_SILU; L.eps = eps; L.bf16 = dtype == SFDA_BF16;
    return sfda::launch_norm_bwd(L, static_cast<hipStream_t>(stream)) == hipSuccess ? SFDA_OK : SFDA_ERR_HIP;
}

}  // extern "C"
