// Which kernel a product on microscaled operands runs.
#include "dfq_host.hpp"

namespace dfq {

namespace {

// Microseconds of a call: fixed + depth * K / 1000 + rounds * (tile + K / 1e6 * (byte * bytes + product * products)), with K in whole
// 256s, rounds the workgroups a compute unit gets, bytes what a workgroup reads of its operands for one k and products its tile's,
// twice for an 8-bit operand and four times for the bfloat16 form that float32 results of one need.  Fitted to 705 calls (1 to 8192
// tokens, 32 to 16384 features, K 64 to 16384, every pair of elements) under every form: each form's times within 12 % of its line in
// the mean, and the form the lines choose 1.027 times the fastest one's time in the mean.  Shapes left out because they were best in
// few calls and by little: 64 x 64 by reductions shared in a workgroup, 64 x 128, 128 x 128 with a deeper ring (0.8 % together).
struct FormTime {
    LinearMxForm form;
    int tokens, features;
    double fixed, tile, depth, byte, product;
};
const FormTime kForms[] = {
    {LinearMxForm::Stream16x16, 16, 16, 4.29, 0.587, 0.0, 11.1, 0.0943},
    {LinearMxForm::Stream16x32, 16, 32, 3.84, 1.01, 0.0, 13.7, 0.0729},
    {LinearMxForm::Stream32x32, 32, 32, 2.88, 2.18, 0.0, 7.1, 0.162},
    {LinearMxForm::Stream32x64, 32, 64, 3.61, 1.52, 0.0, 10.8, 0.108},
    {LinearMxForm::Tile64x64, 64, 64, 3.48, 1.39, 1.03, 2.91, 0.161},
    {LinearMxForm::Tile128x128, 128, 128, 3.35, 3.20, 0.698, 6.50, 0.083},
    {LinearMxForm::Tile256x256, 256, 256, 0.0, 13.3, 0.298, 0.0, 0.0702},
};

double form_time(const FormTime &f, const LinearMxArgs &a)
{
    const double tiles = (double)((a.M + f.tokens - 1) / f.tokens) * ((a.N + f.features - 1) / f.features);
    const double rounds = (double)(long long)((tiles + 255) / 256);
    const int bx = a.elem_x ? 8 : 4, bw = a.elem_w ? 8 : 4;
    const bool wide = bx == 8 || bw == 8, exact = wide && !a.q.codes && a.dtype == 0;
    const double bytes = (f.tokens * bx + f.features * bw) / 8.0, products = (double)f.tokens * f.features * (exact ? 4 : wide ? 2 : 1);
    const double K = (a.K + 255) / 256 * 256;
    return f.fixed + f.depth * K * 1e-3 + rounds * (f.tile + K * 1e-6 * (f.byte * bytes + f.product * products));
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
