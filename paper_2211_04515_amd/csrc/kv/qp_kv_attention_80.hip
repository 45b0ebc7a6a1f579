// Attention over the 4-bit key/value cache with heads of 80 (a file of its own: they compile side by side).
#include "qp_kv_attention.hpp"

namespace qp {
QP_KV_ATTENTION_DIM(80);
}
