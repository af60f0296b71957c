// fa_forward_paged_tree where a sequence's drafts and the heads of a group make 32 rows at most: the streaming kernel of fa_paged.cuh.
#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/fa.h"
#include "fa_handle.h"
#include "fa_paged_host.h"
#include "fa_paged_list.h"

namespace fa_host {

template <int DQK, int DV, bool kE4m3>
static fa_status launch_few(fa_handle* h, int block, const CUtensorMap& mk, const CUtensorMap& mv, fa::PagedParams& p, cudaStream_t st) {
    if (block == 32) return launch_paged<DQK, DV, kE4m3, false, 32, true>(h, mk, mv, p, st);
    return launch_paged<DQK, DV, kE4m3, false, 16, true>(h, mk, mv, p, st);
}

fa_status launch_tree_few(fa_handle* h, int dqk, int dv, bool e4m3, const CUtensorMap& mk, const CUtensorMap& mv, fa::PagedParams& p, cudaStream_t st) {
    set_list(p, dqk, dv, e4m3);
    p.row_blocks = 1;
    const int block = rows_per_block(p.Hq / p.Hkv * p.Sq, dqk, e4m3, false);
    if (dqk == 64) return e4m3 ? launch_few<64, 64, true>(h, block, mk, mv, p, st) : launch_few<64, 64, false>(h, block, mk, mv, p, st);
    if (dqk == 192) return e4m3 ? launch_few<192, 128, true>(h, block, mk, mv, p, st) : launch_few<192, 128, false>(h, block, mk, mv, p, st);
    return e4m3 ? launch_few<128, 128, true>(h, block, mk, mv, p, st) : launch_few<128, 128, false>(h, block, mk, mv, p, st);
}

fa_status plan_tree_few(int num_sms, size_t scratch, fa::PagedParams& p, int dqk, int dv, bool e4m3, fa_paged_plan_info* out, fa_paged_piece* pieces,
                        int max_pieces) {
    return plan_paged(num_sms, scratch, p, dqk, dv, e4m3, false, true, out, pieces, max_pieces);
}

}  // namespace fa_host
