// A block on a device: its tables and workspace.
#include <new>

#include "block.hpp"
#include "common.hpp"

namespace {

void release_device(ccdc_block_t *b)
{
    int cur = -1;
    const bool sw = b->device >= 0 && hipGetDevice(&cur) == hipSuccess && cur != b->device && hipSetDevice(b->device) == hipSuccess;
    if (b->device >= 0) {
        (void)hipFree(b->d_first);
        (void)hipFree(b->d_chunk_first);
        (void)hipFree(b->d_row_of);
        (void)hipFree(b->d_chunks);
        (void)hipFree(b->d_workspace);
        if (b->ws_event) (void)hipEventDestroy((hipEvent_t)b->ws_event);
    }
    if (sw) (void)hipSetDevice(cur);
    b->d_first = b->d_chunk_first = nullptr;
    b->d_row_of = nullptr;
    b->d_chunks = nullptr;
    b->d_workspace = nullptr;
    b->ws_event = b->ws_stream = nullptr;
    b->ws_used = b->uploaded = false;
    b->device = -1;
}

int allocate(void **d, size_t bytes)
{
    if (hipMalloc(d, bytes ? bytes : 1) == hipSuccess) return CCDC_OK;
    (void)hipGetLastError();
    *d = nullptr;
    return CCDC_ENOMEM;
}

template <class E>
int to_device(const std::vector<E> &h, E **d)
{
    const int rc = allocate((void **)d, h.size() * sizeof(E));
    if (rc != CCDC_OK || h.empty()) return rc;
    if (hipMemcpy(*d, h.data(), h.size() * sizeof(E), hipMemcpyHostToDevice) == hipSuccess) return CCDC_OK;
    (void)hipGetLastError();
    return CCDC_EHIP;
}

}  // namespace

extern "C" {

void ccdc_block_destroy(ccdc_block_t *block)
{
    if (!block) return;
    release_device(block);
    delete block;
}

int ccdc_block_bind(ccdc_block_t *block, int files, const int64_t *tokens, const int32_t *ids)
{
    if (!block) return CCDC_EINVAL;
    int rc;
    try {
        rc = ccdc::bind_block(block, files, tokens, ids);
    } catch (const std::bad_alloc &) {
        rc = CCDC_ENOMEM;
    }
    if (rc == CCDC_OK) release_device(block);    // tables of an earlier batch are stale
    return rc;
}

int ccdc_block_upload(ccdc_block_t *block)
{
    if (!block) return CCDC_EINVAL;
    if (!block->bound) return CCDC_ESTATE;
    release_device(block);
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) {
        (void)hipGetLastError();
        return CCDC_EHIP;
    }
    block->device = dev;
    int rc = to_device(block->first, &block->d_first);
    if (rc == CCDC_OK) rc = to_device(block->chunk_first, &block->d_chunk_first);
    if (rc == CCDC_OK) rc = to_device(block->row_of, &block->d_row_of);
    if (rc == CCDC_OK) rc = to_device(block->chunks, &block->d_chunks);
    if (rc == CCDC_OK) rc = allocate(&block->d_workspace, block->workspace_bytes);
    hipEvent_t ev = nullptr;
    if (rc == CCDC_OK && hipEventCreateWithFlags(&ev, hipEventDisableTiming) != hipSuccess) {
        (void)hipGetLastError();
        rc = CCDC_EHIP;
    }
    block->ws_event = ev;
    if (rc != CCDC_OK) {
        release_device(block);
        return rc;
    }
    block->uploaded = true;
    return CCDC_OK;
}

}  // extern "C"
