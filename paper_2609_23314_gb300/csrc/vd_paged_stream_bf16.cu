// vd_paged_stream_bf16.cu -- the streaming attention kernels over bf16 pages.
#include "vd_paged_stream.cuh"

namespace vd {

const PagedKernel kPagedBf16[8][2] = {
    {paged_stream<2, 1, false>(), paged_stream<2, 2, false>()},
    {paged_stream<2, 1, false>(), paged_stream<2, 2, false>()},
    {paged_stream<3, 1, false>(), paged_stream<3, 2, false>()},
    {paged_stream<4, 1, false>(), paged_stream<4, 2, false>()},
    {paged_stream<6, 1, false>(), paged_stream<6, 1, false>()},
    {paged_stream<6, 1, false>(), paged_stream<6, 1, false>()},
    {paged_stream<8, 1, false>(), paged_stream<8, 1, false>()},
    {paged_stream<8, 1, false>(), paged_stream<8, 1, false>()},
};

}  // namespace vd
