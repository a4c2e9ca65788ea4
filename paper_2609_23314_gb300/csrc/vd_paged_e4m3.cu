// vd_paged_e4m3.cu -- the attention kernels over e4m3 pages.
#include "vd_paged_stream.cuh"
#include "vd_paged_tile.cuh"

namespace vd {

const PagedKernel kPagedE4m3[8][3] = {
    {paged_stream<2, 1, true>(), paged_stream<2, 1, true>(), paged_tile<2, true>()},
    {paged_stream<2, 1, true>(), paged_stream<2, 1, true>(), paged_tile<2, true>()},
    {paged_stream<3, 1, true>(), paged_stream<3, 1, true>(), paged_tile<3, true>()},
    {paged_stream<4, 1, true>(), paged_stream<4, 1, true>(), paged_tile<4, true>()},
    {paged_stream<6, 1, true>(), paged_stream<6, 1, true>(), paged_tile<6, true>()},
    {paged_stream<6, 1, true>(), paged_stream<6, 1, true>(), paged_tile<6, true>()},
    {paged_stream<8, 1, true>(), paged_stream<8, 1, true>(), paged_tile<8, true>()},
    {paged_stream<8, 1, true>(), paged_stream<8, 1, true>(), paged_tile<8, true>()},
};

}  // namespace vd
