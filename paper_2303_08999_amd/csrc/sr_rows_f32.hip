// The layers' kernel for very many rows and a weight that registers hold, f32 (sr_rows.h).
#include <type_traits>

#include "sr_rows.h"

namespace srd {
template hipError_t launch_rows<float>(const GemmArgs&, int, hipStream_t);
}  // namespace srd
