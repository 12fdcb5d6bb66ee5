// The kernel of a form.
#pragma once

#include "lif_packed_few.h"
#include "lif_packed_form.h"
#include "lif_packed_many.h"

namespace lif {

// Whether it launched: not every form is compiled for every type and group.
template <typename X, int G, bool ZEROS>
bool launch_product_form(const ProductArgs& a, PackedForm f, hipStream_t s) {
    const int tiles = (a.w.n_out + kTileOut - 1) / kTileOut;
    constexpr bool kF32 = sizeof(X) == 4;
    constexpr int kWide = kF32 ? 2 : 1;
    auto go = [&](auto kernel, int outs, int rows, int waves) {
        hipLaunchKernelGGL(kernel, dim3((tiles + outs - 1) / outs, (a.rows + rows - 1) / rows), dim3(waves * 64), 0, s, a);
        return true;
    };
    switch (f) {
        case PackedForm::few4: return go(k_packed_few<X, G, ZEROS, 1, 4, 8>, 1, 16, 8);
        case PackedForm::few8: return go(k_packed_few<X, G, ZEROS, 2, 4 / kWide, 8>, 1, 16, 8);
        case PackedForm::few16: return go(k_packed_few<X, G, ZEROS, 4, 2 / kWide, 8 / kWide>, 1, 16, 8 / kWide);
        case PackedForm::outs32_rows16: return go(k_packed_many<X, G, ZEROS, 1, 2, 4>, 2, 16, 8);
        case PackedForm::outs128_rows64: return go(k_packed_many<X, G, ZEROS, 4, 8, 1>, 8, 64, 8);
        case PackedForm::outs32_rows16_16:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 1, 2, 8>, 2, 16, 16);
            break;
        case PackedForm::outs32_rows32:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 2, 2, 4>, 2, 32, 8);
            break;
        case PackedForm::outs32_rows32_16:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 2, 2, 8>, 2, 32, 16);
            break;
        case PackedForm::outs48_rows32:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 2, 3, 5>, 3, 32, 15);
            break;
        case PackedForm::outs48_rows48:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 3, 3, 4>, 3, 48, 12);
            break;
        case PackedForm::outs64_rows16:
            if constexpr (kF32) return go(k_packed_many<X, G, ZEROS, 1, 4, 2>, 4, 16, 8);
            break;
        case PackedForm::outs64_rows32_16:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 2, 4, 4>, 4, 32, 16);
            break;
        case PackedForm::outs64_rows32:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 2, 4, 2>, 4, 32, 8);
            break;
        case PackedForm::outs64_rows48:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 3, 4, 2>, 4, 48, 8);
            break;
        case PackedForm::outs64_rows64_16:
            if constexpr (!kF32 && G > 32) return go(k_packed_many<X, G, ZEROS, 4, 4, 4>, 4, 64, 16);
            break;
        case PackedForm::outs64_rows64:
            if constexpr (!kF32 && G > 32) return go(k_packed_many<X, G, ZEROS, 4, 4, 2>, 4, 64, 8);
            break;
        case PackedForm::outs80_rows64:
            if constexpr (!kF32 && G > 32) return go(k_packed_many<X, G, ZEROS, 4, 5, 3>, 5, 64, 15);
            break;
        case PackedForm::outs96_rows32:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 2, 6, 2>, 6, 32, 12);
            break;
        case PackedForm::outs96_rows64:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 4, 6, 2>, 6, 64, 12);
            break;
        case PackedForm::outs112_rows48:
            if constexpr (!kF32) return go(k_packed_many<X, G, ZEROS, 3, 7, 2>, 7, 48, 14);
            break;
    }
    return false;
}
template <typename X>
bool launch_product_as(const ProductArgs& a, PackedForm f, bool zeros, hipStream_t s) {
    if (a.w.group == 32) return zeros ? launch_product_form<X, 32, true>(a, f, s) : launch_product_form<X, 32, false>(a, f, s);
    if (a.w.group == 64) return zeros ? launch_product_form<X, 64, true>(a, f, s) : launch_product_form<X, 64, false>(a, f, s);
    if (a.w.group == 128) return zeros ? launch_product_form<X, 128, true>(a, f, s) : launch_product_form<X, 128, false>(a, f, s);
    return false;
}

}  // namespace lif
