// The scans of linear attention with a decay (decay.hpp) over rows of bf16.
#include "decay.hpp"

namespace nsd {
namespace decay {

nsd_status launch_scan_bf16(Kind kind, const Scan &a, hipStream_t st) {
    return launch_any<Bf16>(kind, a, st);
}

}  // namespace decay
}  // namespace nsd
