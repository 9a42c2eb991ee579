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
        (void)hipFree(b->d_tables);
        (void)hipFree(b->d_workspace);
        if (b->ws_event) (void)hipEventDestroy((hipEvent_t)b->ws_event);
    }
    if (sw) (void)hipSetDevice(cur);
    b->d_first = b->d_chunk_first = nullptr;
    b->d_row_of = nullptr;
    b->d_chunks = nullptr;
    b->d_tables = b->d_workspace = nullptr;
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

// All tables in one allocation and one copy: a block is bound anew for every batch of other lengths, and with four of each that took
// 50 us more.
int to_device(ccdc_block_t *b)
{
    std::vector<char> host;
    const auto put = [&](const auto &table) {
        const size_t at = host.size(), bytes = table.size() * sizeof(table[0]);
        host.resize(at + (bytes + 255) / 256 * 256);
        if (bytes) __builtin_memcpy(host.data() + at, table.data(), bytes);
        return at;
    };
    const size_t first = put(b->first), chunk_first = put(b->chunk_first), row_of = put(b->row_of), chunks = put(b->chunks);
    const int rc = allocate(&b->d_tables, host.size());
    if (rc != CCDC_OK) return rc;
    if (hipMemcpy(b->d_tables, host.data(), host.size(), hipMemcpyHostToDevice) != hipSuccess) {
        (void)hipGetLastError();
        return CCDC_EHIP;
    }
    char *d = static_cast<char *>(b->d_tables);
    b->d_first = reinterpret_cast<int32_t *>(d + first);
    b->d_chunk_first = reinterpret_cast<int32_t *>(d + chunk_first);
    b->d_row_of = reinterpret_cast<ccdc::RowOf *>(d + row_of);
    b->d_chunks = reinterpret_cast<ccdc::Chunk *>(d + chunks);
    return CCDC_OK;
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
    int rc;
    try {
        rc = to_device(block);
    } catch (const std::bad_alloc &) {
        rc = CCDC_ENOMEM;
    }
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
