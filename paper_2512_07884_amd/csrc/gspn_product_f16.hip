// Products with an epilogue (gspn_product_impl.hpp): f16 storage.
#include "gspn_product_impl.hpp"

namespace gspn {
hipError_t launch_product_f16(const ProductParams& p, int form, int outcome, int tile, hipStream_t s) {
    return launch_product_type<f16_t>(p, form, outcome, tile, s);
}
}  // namespace gspn
