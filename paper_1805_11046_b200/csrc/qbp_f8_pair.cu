#include "qbp_f8.cuh"
namespace qbp {
bool f8_pair_eligible(const F8Product &) { return false; }
int launch_f8_pair(const F8Product &, cudaStream_t) { return QBP_ERR_UNSUPPORTED_SHAPE; }
}
