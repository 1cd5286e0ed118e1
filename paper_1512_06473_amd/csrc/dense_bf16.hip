// The dense layers in bfloat16.
#include "dense_kernels.h"

namespace qcnn {
namespace dense {

hipError_t run_bf16(const DenseCall& c, hipStream_t stream) { return dispatch<__bf16>(c, stream); }

}  // namespace dense
}  // namespace qcnn
