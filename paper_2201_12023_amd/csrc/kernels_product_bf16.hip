// The tiled product for one element type (one file each, to build them side by side).
#include "product_kernel.hpp"

namespace alpa {

hipError_t launch_product_bf16(hipStream_t st, Forms forms, Epilogue epi, int tile, const ProductArgs &g)
{
    return launch_forms<bf16>(st, forms, epi, tile, g);
}

}  // namespace alpa
