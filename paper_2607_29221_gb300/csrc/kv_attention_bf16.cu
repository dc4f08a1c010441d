#include "kv_attention_impl.cuh"

namespace mosaic {
MOSAIC_ATTEND_TYPE(__nv_bfloat16, with_instance<__nv_bfloat16>)
}
