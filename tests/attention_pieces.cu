// How the attention kernels deal out their work, on the host.
#include "attention_shared.cuh"

// blocks that prepare the gradients, of a device of `sms`
extern "C" long long run_prepare_blocks(int causal, int n_seg, long long rows, int heads, int lanes, int sms) {
    tiga::AttnParams p{};
    p.causal = causal;
    p.n_seg = n_seg;
    p.heads = heads;
    return tiga::prepare_blocks(p, rows * heads, lanes, sms);
}
