// vd_paged_stream_e4m3.cu -- the streaming attention kernels over e4m3 pages.
#include "vd_paged_stream.cuh"

namespace vd {

const PagedKernel kPagedE4m3[8][2] = {
    {paged_stream<2, 1, true>(), paged_stream<2, 2, true>()},
    {paged_stream<2, 1, true>(), paged_stream<2, 2, true>()},
    {paged_stream<3, 1, true>(), paged_stream<3, 2, true>()},
    {paged_stream<4, 1, true>(), paged_stream<4, 2, true>()},
    {paged_stream<6, 1, true>(), paged_stream<6, 1, true>()},
    {paged_stream<6, 1, true>(), paged_stream<6, 1, true>()},
    {paged_stream<8, 1, true>(), paged_stream<8, 1, true>()},
    {paged_stream<8, 1, true>(), paged_stream<8, 1, true>()},
};

}  // namespace vd
