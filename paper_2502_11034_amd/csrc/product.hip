// The products with a plain result of the operators' backward passes, both types, Y along and across k, and parts of the others (product_device.h).
#include "product_device.h"

namespace adagc {
namespace product {
template int run_plain<float, false>(PlainArgs, hipStream_t);
template int run_plain<float, true>(PlainArgs, hipStream_t);
template int run_plain<uint16_t, false>(PlainArgs, hipStream_t);
template int run_plain<uint16_t, true>(PlainArgs, hipStream_t);
template int lay<float>(const LaySource*, int, int64_t, const Layout&, hipStream_t);
template int lay<uint16_t>(const LaySource*, int, int64_t, const Layout&, hipStream_t);
template void launch_parts<Small, uint16_t, false>(const AlongArgs&, hipStream_t);
template void launch_parts<Small, uint16_t, true>(const AlongArgs&, hipStream_t);
template void launch_parts<Staged<uint16_t>, uint16_t, false>(const AlongArgs&, hipStream_t);
template void launch_parts<Staged<uint16_t>, uint16_t, true>(const AlongArgs&, hipStream_t);
template void launch_parts<Slim, float, false>(const AlongArgs&, hipStream_t);
template void launch_parts<Slim, float, true>(const AlongArgs&, hipStream_t);
template void launch_parts<Staged<float>, float, false>(const AlongArgs&, hipStream_t);
template void launch_parts<Staged<float>, float, true>(const AlongArgs&, hipStream_t);
}  // namespace product
}  // namespace adagc
