// The decode step over all of a sequence's pages or over listed ones: the kernel and its launch are paged_decode.h's, where the mathematics and what
// bounds it are.
#include "paged_decode.h"

namespace sablock {

bool decode_paged_supported(const PageDims &d) { return d.G <= 16 && d.D % (d.dtype == SABLOCK_F32 ? 16 : 32) == 0; }

size_t decode_paged_ws_bytes(const PageDims &d) { return decode_ws_bytes_of(d); }

hipError_t launch_decode_paged(const PageDims &d, const void *q, const PageView &pv, const int32_t *list, int32_t n_listed, float *out,
                               void *ws, hipStream_t st)
{
    DecodePagedArgs a;
    return launch_decode_of(a, d, q, pv, list, n_listed, out, ws, st);
}

}  // namespace sablock
