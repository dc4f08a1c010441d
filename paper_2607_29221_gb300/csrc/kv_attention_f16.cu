#include "kv_attention_impl.cuh"

namespace mosaic {
MOSAIC_ATTEND_TYPE(__half, with_instance<__half>)
}
