#include "gated_ffn_mma.cuh"

namespace cdma {
namespace mma {

template cudaError_t launch_all<float>(const FfnProblem&, bool, const LaunchCtl&, cudaStream_t);

}  // namespace mma
}  // namespace cdma
