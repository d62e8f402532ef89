// Which form a microscaled product runs in, and how: arithmetic on sizes, on
// the host alone.
#pragma once
#include <algorithm>
#include <cmath>
#include <cstdint>

namespace quick {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Rows and values of activations that a product's own launch quantises: a
// workgroup does it all, so it has to stay small beside its weights, and its
// codes, with the sums of two column tiles, within 64 KiB of LDS.
constexpr int kFusedRows = 4;
constexpr int64_t kFusedValues = 57344;

inline bool fused_quantisation(int64_t M, int64_t K) { return M <= kFusedRows && M * K <= kFusedValues; }

// The forms of the product, and what a call in each takes (us):
//   pipe   = start + max(KS * alone, tiles * (KS * shared + turn))
//   memory = 2 + bytes of weights / stream,   time = (pipe^4 + memory^4)^(1/4)
// with KS steps of 128 channels and the tiles of the busiest of 256 compute
// units: `shared` is a step's share of the unit, `turn` what a tile takes
// besides its steps, `alone` a step's latency where the unit has one tile.  A
// stream form's `shared` counts column tiles plus activations (`rows` of a
// column tile's cost for 16 rows).  Fitted to the times of all forms on 702
// sizes (1 to 2048 rows, 512 to 57344 columns, 512 to 28672 channels, weights
// from HBM) without leading workgroups: 8 to 24 % (rms) a form over all of
// them.  Past 4e11 operations, where the clock falls, the three largest forms
// take 1.3 to 1.4 times what it says (2048 x 57344 x 8192: 457 us, 293 by it),
// all of them, so that the order holds: of 21 such sizes the form chosen is at
// most 0.8 % slower than the fastest.  Over all sizes, with leading workgroups,
// that is 0.5 % on average and 26 % at most (fitting anew gives 0.4).  Over
// experts, whose rows are taken as equal, it was 0 to 11 % on nine sizes (8192
// rows over 32 experts of 5760 x 2880: 179 us, 162 in 128 x 256).
struct Form {
    int bm, bn;    // rows and columns of a tile
    float start, alone, shared, turn, stream, rows;
};
constexpr int kFormCount = 10;
constexpr Form kForms[kFormCount] = {
    {16, 16, 3.05f, 0.0139f, 0.0265f, 0.453f, 5.26f, 1.52f},    // stream forms
    {16, 32, 2.94f, 0.0428f, 0.0166f, 0.943f, 5.08f, 2.90f},
    {16, 64, 2.59f, 0.0f, 0.0161f, 1.120f, 4.27f, 3.15f},
    {32, 128, 1.12f, 0.1902f, 0.1602f, 1.55f, 5.55f, 0.0f},     // tiled forms
    {64, 64, 2.04f, 0.0f, 0.1263f, 1.03f, 5.84f, 0.0f},         // eight stages
    {64, 128, 0.11f, 0.0f, 0.1862f, 3.24f, 5.18f, 0.0f},        // eight stages
    {64, 128, 1.68f, 0.2126f, 0.2049f, 1.08f, 5.49f, 0.0f},
    {128, 128, 1.78f, 0.2444f, 0.2573f, 1.48f, 4.26f, 0.0f},
    {128, 256, 0.0f, 0.2039f, 0.3873f, 4.31f, 4.16f, 0.0f},
    {256, 256, 0.0f, 0.6207f, 0.5595f, 6.07f, 4.00f, 0.0f},
};

// A product of M rows with one of E matrices each, [N][K].
struct MxSizes {
    int64_t M, N, K, E;
    bool grouped, gated;
    bool x16;      // 16-bit activations, which the launch quantises
};

inline bool is_stream(const Form& f) { return f.bm == 16; }

// Whether a form is built for a call.
inline bool form_takes(const Form& f, const MxSizes& s)
{
    // a gate tile and its up tile in one wave
    if (s.gated && f.bn < 32) return false;
    // quantisation on the way, in the narrow stream forms
    if (s.x16 && (s.grouped || !is_stream(f) || f.bn > 32)) return false;
    // a tail of channels: the largest form's accumulators leave no registers for it
    return s.K % 128 == 0 || f.bm * f.bn < 65536;
}

inline double form_cost(const Form& f, double tiles, double rows, int64_t KS, double bytes)
{
    double shared = f.shared;
    if (is_stream(f)) shared *= f.bn / 16 + f.rows * std::min(rows, 16.0) / 16;
    const double pipe = f.start + std::max(KS * (double)f.alone, std::ceil(tiles / 256) * (KS * shared + f.turn));
    const double memory = 2.0 + bytes / (f.stream * 1e6);
    return pipe * pipe * pipe * pipe + memory * memory * memory * memory;
}

// Experts that have rows, as far as is known on the host; rows of each.
inline int64_t busy_experts(const MxSizes& s) { return s.grouped ? std::min(s.E, s.M) : 1; }
inline double expert_rows(const MxSizes& s) { return (double)s.M / busy_experts(s); }

// The cheapest of the forms that take the call.
template <int COUNT>
int choose_form(const Form (&forms)[COUNT], const MxSizes& s)
{
    const int64_t busy = busy_experts(s);
    const double rows = expert_rows(s);
    int best = -1;
    double least = 0;
    for (int i = 0; i < COUNT; i++) {
        const Form& f = forms[i];
        if (!form_takes(f, s)) continue;
        // an expert's last tile is half empty on average
        const double high = busy > 1 ? std::max(1.0, rows / f.bm + 0.5) : std::ceil(rows / f.bm);
        const double tiles = high * busy * ceil_div(s.N, f.bn);
        const double c = form_cost(f, tiles, rows, ceil_div(s.K, 128), (double)busy * s.N * s.K * 17 / 32);
        if (best < 0 || c < least) {
            best = i;
            least = c;
        }
    }
    return best;
}

// Whether the weights come past the caches: where a tile of rows reads them
// once, and they do not stay in the 256 MB cache from call to call anyway
// (70B gate+up, 16 rows: 39.3 us, 42.5 through them; but 7B down, 23 MB and 16
// rows, 10.5 against 8.0 where a call finds what the one before has left).
constexpr int64_t kOnceBytes = (int64_t)192 << 20;

inline bool weights_once(const MxSizes& s, int bm)
{
    return bm <= 64 && expert_rows(s) <= bm && std::min(s.E, s.M) * s.N * s.K / 2 >= kOnceBytes;
}

// Whether every column tile gets a leading workgroup.  Where the row tiles of a
// column run in step, and none is light, all of them wait for the same weights
// at a time; behind one that is ahead they find them in L2 (128 x 4096 x 11008
// 20.8 -> 14.0 us, 64 x 8192 x 28672 50.5 -> 37.4, 512 x 5120 x 13824 43.7 ->
// 31.9, 1536 x 8192 x 28672 193 -> 180, weights from HBM; with 1024 channels no
// difference).  There has to be room for it: past one workgroup a compute unit
// (64 x 12288 x 4096, from 192 to 384: 10.5 -> 11.8; 1024 x 8192 x 8192, from
// 256 to 288: 42.7 -> 61.7), or where wide tiles pass half of the units (256 x
// 4096 x 11008, from 128 to 160: 20.2 -> 26.0), it costs more than it gives.
inline bool has_lead(const MxSizes& s, int64_t tiles, int64_t columns, const Form& f)
{
    const int64_t light = s.M % f.bm;
    const bool crosses = f.bn > 64 && tiles <= 128 && tiles + columns > 128;
    return s.K >= 2048 && (light == 0 || light > f.bm / 4) && tiles + columns <= 256 && !crosses;
}

struct MxPlan {
    int form;
    bool tail, once;               // K % 128 != 0; the weights come past the caches
    int lead;                      // 1: a leading workgroup for each column tile
    int64_t row_tiles, columns;    // at most; column tiles (runs of them, in a stream form)
};

inline MxPlan plan_product(const MxSizes& s)
{
    MxPlan p = {choose_form(kForms, s), false, false, 0, 0, 0};
    if (p.form < 0) return p;    // none takes the call
    const Form& f = kForms[p.form];
    p.tail = s.K % 128 != 0;
    p.once = weights_once(s, f.bm);
    p.row_tiles = s.grouped ? s.M / f.bm + std::min(s.E, s.M) : ceil_div(s.M, f.bm);
    p.columns = ceil_div(s.N, f.bn);
    p.lead = !s.grouped && !is_stream(f) && has_lead(s, p.row_tiles * p.columns, p.columns, f);
    return p;
}

}  // namespace quick
