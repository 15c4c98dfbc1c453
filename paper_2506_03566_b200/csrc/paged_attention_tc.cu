#include "paged_attention.cuh"
bool paged_attn_tc_supported(const poss_page_pool&, float) { return false; }
size_t paged_attn_tc_workspace(const poss_page_pool&, int, int, int, int) { return 0; }
void launch_paged_attn_tc(Launcher& L, const PagedAttnArgs&, const void*, const poss_page_pool&) { L.err = POSS_E_SHAPE; }
