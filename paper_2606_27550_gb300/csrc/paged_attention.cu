// paged_attention.cu -- tree attention over pages of 16 bits (paged_attention.cuh).
#include "paged_attention.cuh"

namespace tv {

TB_BOUNDS_COUNTER(bounds_violations_paged_attention)

}  // namespace tv

using namespace tv;

extern "C" tb_status paged_tree_attention(const tb_bank *bank, const tb_requests *req, const tb_pages *pages,
                                          int layer, const void *plan, size_t plan_bytes, const void *q, int n_rows,
                                          int n_q_heads, float scale, float softcap, const float *slopes, void *out,
                                          float *lse, void *workspace, size_t workspace_bytes, tb_stream stream)
{
    const auto fill = [&](PagedArgs &a, int layer) {
        const char *err = nullptr;
        const int box = pages->page_size < kTileKeys ? pages->page_size : kTileKeys;
        const long long off = (long long)layer * pages->layer_stride;
        (void)(make_tmap_pages(&a.tk, pages, static_cast<uint16_t *>(pages->k) + off, box, &err) &&
               make_tmap_pages(&a.tv, pages, static_cast<uint16_t *>(pages->v) + off, box, &err));
        return err;
    };
    return attend<false>(bank, req, pages, layer, plan, plan_bytes, q, n_rows, n_q_heads, scale, softcap, slopes, out,
                         lse, workspace, workspace_bytes, stream, "paged_tree_attention", check_pages, fill);
}
