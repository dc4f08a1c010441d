#include "kv_attention_impl.cuh"

namespace mosaic {
MOSAIC_ATTEND_TYPE(float, with_instance<float>)
}
