#include "cg_internal.h"
extern "C" size_t cg_attn_workspace_bytes(const cg_attn_desc *, int) { return 0; }
extern "C" int cg_attn_fwd(const cg_attn_desc *, const void *, const void *, const void *, const int32_t *, const int32_t *, const float *, void *, float *, void *, void *, size_t, void *) { return CG_EUNSUPPORTED; }
extern "C" int cg_attn_bwd(const cg_attn_desc *, const void *, const void *, const void *, const void *, const int32_t *, const int32_t *, const float *, const void *, const void *, const float *, void *, void *, void *, float *, void *, size_t, void *) { return CG_EUNSUPPORTED; }
