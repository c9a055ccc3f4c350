// The scans of linear attention with a decay (decay.hpp) over rows of fp32.
#include "decay.hpp"

namespace nsd {
namespace decay {

nsd_status launch_scan_f32(Kind kind, const Scan &a, hipStream_t st) {
    return launch_any<float>(kind, a, st);
}

}  // namespace decay
}  // namespace nsd
