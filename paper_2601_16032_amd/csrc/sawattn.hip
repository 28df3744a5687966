// libsawattn.so, all of it: one translation unit, so that the library holds one code object.
#include "attn_fwd.hip"

#include "paged.h"

#include "attn_pages.hip"
#include "attn_prepare.hip"
#include "attn_decode.hip"
#include "attn_fork.hip"
#include "attn_shared.hip"
