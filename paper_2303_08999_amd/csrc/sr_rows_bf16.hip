// The layers' kernel for very many rows and a weight that registers hold, bf16 (sr_rows.h).
#include <type_traits>

#include "sr_rows.h"

namespace srd {
template hipError_t launch_rows<bf16raw>(const GemmArgs&, int, hipStream_t);
}  // namespace srd
