// The host side of the calls on a cache in 4 bits on randomised inputs, for a build
// with AddressSanitizer and UndefinedBehaviorSanitizer: the decode split with its
// workspace, and the prefill's choice of pieces (the source is included for its
// planner).  Nothing here launches a kernel or touches a GPU: the device pointers are
// host addresses the planners only check for alignment.  Prints "ok" when every
// check holds.
#include <cstdio>
#include <vector>

#include "kv4_prefill.hip"

namespace {

uint64_t g_state = 0x2545F4914F6CDD1Dull;
uint32_t next_u32() {  // xorshift64*
    g_state ^= g_state >> 12;
    g_state ^= g_state << 25;
    g_state ^= g_state >> 27;
    return static_cast<uint32_t>((g_state * 0x9E3779B97F4A7C15ull) >> 32);
}
int uniform(int lo, int hi) { return lo + static_cast<int>(next_u32() % static_cast<uint32_t>(hi - lo + 1)); }
int spread(int bits) { return static_cast<int>(next_u32() % (1u << uniform(1, bits))); }

int g_fail = 0;
void check(bool ok, const char *what, int it) {
    if (!ok) {
        std::fprintf(stderr, "check failed at iteration %d: %s (%s)\n", it, what, mw_last_error());
        ++g_fail;
    }
}

alignas(256) unsigned char g_fake[4096];  // stands in for device buffers: never dereferenced

void decode() {
    int short_units = 0;
    for (int it = 0; it < 3000; ++it) {
        const int hkv = 1 << uniform(0, 3), group = uniform(1, 16), batch = uniform(0, 3) ? uniform(1, 8) : uniform(1, 300);
        mw_kv_pool_desc desc{1 << 14, 16, hkv, 128};
        mw_kv_pool *pool = nullptr;
        check(mw_kv4_pool_create(&desc, g_fake, g_fake, g_fake, &pool) == MW_OK, "pool create", it);
        const mw_attn_shape shape{hkv * group, hkv, 128, 0.0883883f};
        std::vector<int32_t> lens(batch);
        for (int32_t &n : lens) n = 1 + spread(17);
        size_t bytes = 0;
        check(mw_kv4_decode_workspace_size(&shape, batch, lens.data(), &bytes) == MW_OK, "size", it);
        int32_t *const p = reinterpret_cast<int32_t *>(g_fake);
        mw_decode_args a{pool, shape, batch, lens.data(), p, p, 1 << 13, g_fake, g_fake, g_fake, bytes, 0};
        const int cus = uniform(1, 256);
        DecodePlan pl;
        check(decode_prepare(&a, cus, &pl, "decode", true) == MW_OK, "the size covers the split of every CU count", it);
        int64_t pages = 0, most = 0;  // segments padded to steps of four pages
        for (int32_t n : lens) {
            pages += (n + 63) / 64 * 4;
            most = std::max<int64_t>(most, (n + 15) / 16);
        }
        check(pl.units * pl.per_unit >= pl.total && (pl.units - 1) * pl.per_unit < pl.total,
              "units cover the pages", it);
        check(pl.aligned || (pl.total == pages * hkv && pl.per_unit % 4 == 0), "pages of a balanced split", it);
        check(pl.slots >= pl.units && pl.off_meta + static_cast<size_t>(pl.slots) * 4 <= pl.bytes, "slots and flags", it);
        check(pl.units <= cus, "a unit per CU at most", it);
        if (!pl.aligned && pl.units > 1)  // short units only where they leave few pieces
            check(pl.per_unit >= (most <= 512 ? 9 : 17), "pages of a unit", it);
        short_units += pl.units > 1 && pl.per_unit < 32;
        if (bytes > 256) {
            a.workspace_bytes = pl.bytes - 1;
            check(decode_prepare(&a, cus, &pl, "decode", true) == MW_ERR_INVALID_ARG, "a short workspace", it);
        }
        mw_kv_pool_destroy(pool);
    }
    check(short_units > 100, "short units occur", short_units);
}

void prefill() {
    int few = 0, many = 0, split = 0;
    for (int it = 0; it < 20000; ++it) {
        const int hkv = 1 << uniform(0, 5), group = uniform(1, it % 8 ? 16 : 300), batch = uniform(0, 2) ? uniform(1, 6) : uniform(1, 200);
        std::vector<int32_t> n(batch), r(batch);
        for (int b = 0; b < batch; ++b) {
            n[b] = uniform(0, 7) ? std::min(spread(10), uniform(1, 1100) / group) : spread(9);
            r[b] = uniform(0, 2) ? spread(15) : it % 16 ? 0 : spread(22);
        }
        const FewPlan p = few_plan(batch, n.data(), r.data(), hkv, group);
        size_t bytes = 0;
        const mw_attn_shape shape{hkv * group, hkv, 128, 0.0883883f};
        check(mw_kv4_prefill_workspace_size(&shape, batch, n.data(), r.data(), 0, &bytes) == MW_OK, "size", it);
        if (p.groups == 0) {
            ++many;
            continue;
        }
        ++few;
        check(bytes == p.bytes, "the size is the plan's", it);
        check(p.piece_tiles >= 1 && p.piece_tiles <= kTableTiles && p.max_pieces >= 1 && p.max_pieces <= kMaxPieces, "pieces", it);
        int64_t groups = 0;
        for (int b = 0; b < batch; ++b) {  // as the kernels count them
            if (n[b] == 0) continue;
            const int64_t rows = static_cast<int64_t>(n[b]) * group, blocks = (rows + kBlockRows - 1) / kBlockRows;
            check(blocks <= kFewBlocks && std::min<int64_t>(rows, kBlockRows) <= p.block_rows, "blocks of a sequence", it);
            const int tiles = (r[b] + n[b] + kTileKeys - 1) / kTileKeys;
            const int pieces = prefill_pieces(tiles, p.piece_tiles, p.max_pieces);
            groups += blocks * pieces * hkv;
            check(tiles <= p.piece_tiles * p.max_pieces, "tiles of a sequence", it);
            for (int64_t q = 0; q < blocks; ++q) {
                const int nt = prefill_block_tiles<int>(r[b], n[b], static_cast<int>(q), kBlockRows, group);
                const int k = prefill_pieces(nt, p.piece_tiles, p.max_pieces);
                check(nt >= 1 && nt <= tiles && k <= pieces, "pieces of a block", it);
                check(k == 1 || p.rows > 0, "several pieces have a workspace", it);
                for (int i = 0; i < k; ++i)
                    check((i + 1) * nt / k > i * nt / k && (i + 1) * nt / k - i * nt / k <= kTableTiles, "tiles of a piece", it);
            }
        }
        check(groups == p.groups, "a work-group for every block of every piece", it);
        check(p.max_pieces == 1 || p.rows == static_cast<size_t>(groups) * p.block_rows, "a row of the workspace for each of theirs", it);
        check(p.bytes == p.rows * kRowBytes, "bytes of the workspace", it);
        split += p.max_pieces > 1;
    }
    check(few > 1000 && many > 1000 && split > 500, "calls of every kind", few);
}

// Sizes of calls far past any pool.
void prefill_sizes() {
    const int32_t most = INT32_MAX - 64;
    for (int it = 0; it < 200; ++it) {
        const int group = uniform(1, 64);
        const mw_attn_shape shape{group, 1, 128, 0.0883883f};
        const int32_t n = it < 8 ? most : it % 2 ? uniform(1 << 24, most) : 1;
        const int32_t r = n == most ? 0 : uniform(0, most - n);
        size_t bytes = 0;
        check(mw_kv4_prefill_workspace_size(&shape, 1, &n, &r, 0, &bytes) == MW_OK, "size", it);
        check(bytes >= (static_cast<size_t>(n) + r) / 16 * 8192 || (n == 1 && r <= kTableTiles * kMaxPieces * kTileKeys), "bytes", it);
    }
    const mw_attn_shape shape{8, 8, 128, 0.0883883f};
    std::vector<int32_t> n(64, 1 << 30), r(64, 1 << 30);
    size_t bytes = 0;
    check(mw_kv4_prefill_workspace_size(&shape, 64, n.data(), r.data(), 0, &bytes) == MW_ERR_INVALID_ARG, "2^31 tokens", 0);
    for (int32_t &x : r) x -= 100;
    check(mw_kv4_prefill_workspace_size(&shape, 64, n.data(), r.data(), 0, &bytes) == MW_ERR_UNSUPPORTED, "too many pages", 0);
}

}  // namespace

int main() {
    decode();
    prefill();
    prefill_sizes();
    if (g_fail == 0) std::puts("ok");
    return g_fail != 0;
}
