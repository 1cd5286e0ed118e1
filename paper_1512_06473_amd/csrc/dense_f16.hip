// The dense layers in fp16.
#include "dense_kernels.h"

namespace qcnn {
namespace dense {

hipError_t run_f16(const DenseCall& c, hipStream_t stream) { return dispatch<_Float16>(c, stream); }

}  // namespace dense
}  // namespace qcnn
