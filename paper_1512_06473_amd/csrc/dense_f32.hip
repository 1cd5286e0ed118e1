// The dense layers in fp32.
#include "dense_kernels.h"

namespace qcnn {
namespace dense {

hipError_t run_f32(const DenseCall& c, hipStream_t stream) { return dispatch<float>(c, stream); }

}  // namespace dense
}  // namespace qcnn
