// Which kernel a product on microscaled operands runs.
#include "dfq_host.hpp"

namespace dfq {

namespace {

// Microseconds of a call: fixed + rounds * (tile + depth * K / 1000) + load * K / 1e6 * (byte * bytes + product * products), with K in
// whole 256s, rounds the workgroups that a compute unit gets at most and load the same, bytes what a workgroup reads of its operands
// for one k and products its tile's, twice for an aligned 8-bit operand and four times for the bfloat16 form.
// `shared`: two workgroups of a compute unit overlap, so that load is nearer to what the units get in the mean.  Fitted to 1892 calls
// (1 to 8192 tokens, 32 to 16384 features, K 64 to 16384; 4 by 4, 8 by 4 and 8 by 8 bits, the last two aligned and not) under every
// form that could be near: each form's times within 7 to 14 % of its line in the mean, and the form the lines choose 1.024 times the
// fastest one's time in the mean (calls of 8 us and more: 1.016).  Other calls: 423 of 8 by 4, 8 by 8 and 4 by 8 bits 1.019, 141 of
// 4 by 8 aligned 1.011.
struct FormTime {
    LinearMxForm form;
    int tokens, features;
    double fixed, tile, depth, byte, product;
    bool shared;
};
const FormTime kForms[] = {
    {LinearMxForm::Stream16x16, 16, 16, 4.21, 0.600, 0.0, 11.2, 0.0980, false},
    {LinearMxForm::Stream16x32, 16, 32, 3.82, 0.998, 0.0, 13.6, 0.0750, false},
    {LinearMxForm::Stream32x32, 32, 32, 2.91, 2.14, 0.0, 7.11, 0.167, false},
    {LinearMxForm::Stream32x64, 32, 64, 3.72, 1.42, 0.0, 11.0, 0.105, false},
    {LinearMxForm::Tile64x64, 64, 64, 4.27, 0.751, 0.262, 1.71, 0.183, false},
    {LinearMxForm::Tile64x128, 64, 128, 2.99, 2.65, 0.446, 1.75, 0.130, false},
    {LinearMxForm::Tile128x128, 128, 128, 4.15, 1.92, 0.370, 7.00, 0.0930, true},
    {LinearMxForm::Tile128x128Deep, 128, 128, 0.846, 5.15, 0.270, 0.0, 0.105, false},
    {LinearMxForm::Tile256x256, 256, 256, 0.0, 11.8, 0.638, 0.046, 0.0670, false},
};

double form_time(const FormTime &f, const LinearMxArgs &a)
{
    const double tiles = (double)((a.M + f.tokens - 1) / f.tokens) * ((a.N + f.features - 1) / f.features);
    const double rounds = (double)(long long)((tiles + 255) / 256);
    double load = rounds;
    if (f.shared) {
        load = 0.3 * rounds + 0.7 * tiles / 256;
        if (load < 1) load = 1;
    }
    const int bx = a.elem_x ? 8 : 4, bw = a.elem_w ? 8 : 4;
    const bool wide = bx == 8 || bw == 8;
    const double bytes = (f.tokens * bx + f.features * bw) / 8.0, products = (double)f.tokens * f.features * (a.exact() ? 4 : wide ? 2 : 1);
    const double K = (a.K + 255) / 256 * 256;
    return f.fixed + rounds * (f.tile + f.depth * K * 1e-3) + load * K * 1e-6 * (f.byte * bytes + f.product * products);
}

}  // namespace

bool linear_mx_supports(const LinearMxArgs &a, LinearMxForm form)
{
    if (form == LinearMxForm::Direct) return true;
    if (form == LinearMxForm::Stream16x16 && a.q.codes) return false;      // a workgroup has half of a block
    constexpr size_t most = (size_t)1 << 22;                               // 31-bit offsets inside a tile of 256 rows
    return a.ldx <= most && a.ldw <= most && a.ldxs <= most && a.ldws <= most;
}

LinearMxForm linear_mx_select(const LinearMxArgs &a)
{
    LinearMxForm best = LinearMxForm::Direct;
    double least = 0;
    for (const FormTime &f : kForms) {
        if (!linear_mx_supports(a, f.form)) continue;
        const double t = form_time(f, a);
        if (best == LinearMxForm::Direct || t < least) {
            best = f.form;
            least = t;
        }
    }
    return best;
}

hipError_t launch_linear_mx(const LinearMxArgs &a, LinearMxForm form, hipStream_t st)
{
    if (form == LinearMxForm::Auto) form = linear_mx_select(a);
    if (form == LinearMxForm::Direct) return launch_linear_mx_direct(a, st);
    return form < LinearMxForm::Tile64x64 ? launch_linear_mx_stream(a, form, st) : launch_linear_mx_tiles(a, form, st);
}

}  // namespace dfq
