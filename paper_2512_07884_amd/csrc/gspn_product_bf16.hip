// Products with an epilogue (gspn_product_impl.hpp): bf16 storage.
#include "gspn_product_impl.hpp"

namespace gspn {
hipError_t launch_product_bf16(const ProductParams& p, int form, int outcome, int tile, hipStream_t s) {
    return launch_product_type<bf16_t>(p, form, outcome, tile, s);
}
}  // namespace gspn
