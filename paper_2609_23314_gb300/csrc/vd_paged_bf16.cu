// vd_paged_bf16.cu -- the attention kernels over bf16 pages.
#include "vd_paged_stream.cuh"
#include "vd_paged_tile.cuh"

namespace vd {

const PagedKernel kPagedBf16[8][3] = {
    {paged_stream<2, 1, false>(), paged_stream<2, 2, false>(), paged_tile<2, false>()},
    {paged_stream<2, 1, false>(), paged_stream<2, 2, false>(), paged_tile<2, false>()},
    {paged_stream<3, 1, false>(), paged_stream<3, 2, false>(), paged_tile<3, false>()},
    {paged_stream<4, 1, false>(), paged_stream<4, 2, false>(), paged_tile<4, false>()},
    {paged_stream<6, 1, false>(), paged_stream<6, 1, false>(), paged_tile<6, false>()},
    {paged_stream<6, 1, false>(), paged_stream<6, 1, false>(), paged_tile<6, false>()},
    {paged_stream<8, 1, false>(), paged_stream<8, 1, false>(), paged_tile<8, false>()},
    {paged_stream<8, 1, false>(), paged_stream<8, 1, false>(), paged_tile<8, false>()},
};

}  // namespace vd
