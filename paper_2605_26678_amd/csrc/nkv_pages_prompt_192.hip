// nkv_pages_prompt_attention for head dim 192: a source of its own, so that the head dims compile side by side.
#include "nkv_pages_prompt_tile.h"

namespace nkv {
template hipError_t launch_prompt_tiles<192>(const PromptArgs &, const nkv_pages &, hipStream_t);
}
