// The ring through which a block's items go from the warp that finds them to the others, on its own: two warps that meet at every item,
// and a third that stops taking part after `stop` items.
#include "attention_tiles.cuh"

namespace {

struct Numbers {                // hands out items 0 .. total - 1
    tiga::Segment g;
    int s, h, t, steps, i0, i1, total;
    __device__ bool next(const tiga::AttnParams&) { return ++s < total; }
};

// taken[w][0]: items that warp w took; taken[w][1]: the sum of their numbers
__global__ void ring_kernel(const tiga::AttnParams p, int total, int stop, int slow, long long limit, int* taken) {
    __shared__ tiga::ItemRing ring;
    const int warp = threadIdx.x / 32;
    if (threadIdx.x == 0) {
        tiga::items_init(ring, 3);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (warp == 3) {
        if (threadIdx.x % 32 == 0) {
            Numbers it{{0, 0, 0, 0}, 0, 0, 0, 1, 0, 1, total};
            tiga::items_hand_out(ring, p, it, total > 0, limit);
        }
        __syncwarp();
    } else {
        int count = 0, sum = 0;
        for (uint32_t n = 0; warp < 2 || (int)n < stop; ++n) {
            const tiga::Item& e = tiga::item_take(ring, n);
            if (e.steps == 0) break;
            ++count;
            sum += e.s;
            if (warp == 1 && slow) __nanosleep(200000);
            if (warp < 2) asm volatile("bar.sync 1, 64;" ::: "memory");
            tiga::item_return(ring, n);
        }
        if (threadIdx.x % 32 == 0) { taken[2 * warp] = count; taken[2 * warp + 1] = sum; }
    }
}

}  // namespace

extern "C" int run_ring(int total, int stop, int slow, long long limit, int* taken) {
    ring_kernel<<<1, 128>>>(tiga::AttnParams{}, total, stop, slow, limit, taken);
    return (int)cudaGetLastError();
}
