// Entry points of the products with matrices in 4 bits: argument checks, and dispatch to the kernels of linear_*.hip.
#include <algorithm>

#include "linear.hpp"

#define BF_HIP(call)                                                   \
    do {                                                               \
        hipError_t e_ = (call);                                        \
        if (e_ != hipSuccess) return bf::record_hip_error(e_, #call);  \
    } while (0)

namespace {

bool spec_ok(const bifeat_linear_spec *s) {
    return s && s->out_features >= 1 && s->out_features <= (1 << 20) && s->in_features >= 1 && s->in_features <= (1 << 20) &&
           (s->group == 32 || s->group == 64 || s->group == 128) && s->experts >= 1 && s->experts <= 1024;
}

bool type_ok(int32_t d) { return d == BIFEAT_F32 || d == BIFEAT_F16 || d == BIFEAT_BF16; }
bool data_ok(const void *p, int32_t dtype) { return p && (uintptr_t)p % (dtype == BIFEAT_F32 ? 4 : 2) == 0; }

bf::Matrices matrices_of(const bifeat_linear_spec *s, const uint8_t *packed) {
    const int rows = (s->out_features + 15) / 16, blocks = (s->in_features + 127) / 128;
    return {packed, (int64_t)rows * blocks * (1024 + 64 * (128 / s->group)), s->out_features, s->in_features, rows, blocks, s->experts};
}

int64_t sum_bytes(const bifeat_linear_spec *s, int64_t rows) {  // (a multiple of 16)
    return (rows * ((s->in_features + 127) / 128 * (128 / s->group)) + 1) / 2 * 16;
}

// How a product of rows with one matrix is taken.
struct Plan {
    bool many;
    int tb, r, split;
    // the workspace: parts of the sums, then the sums of x
    int64_t parts_bytes(const bifeat_linear_spec *s, int64_t rows) const { return split > 1 ? (split * rows * s->out_features + 3) / 4 * 16 : 0; }
    int64_t bytes(const bifeat_linear_spec *s, int64_t rows) const { return parts_bytes(s, rows) + (many ? sum_bytes(s, rows) : 0); }
};
// Of the ways to take the rows the one that is the fastest by what they measured (bf16, in parentheses fp32; us; 256 workgroups run at a time, for 128 rows 512).
// What the codes take from memory is the same in all of them and not in the figures, which therefore compare ways and foretell no time: one row by 8192 x 28 672
// is 17.9 by them, 29.2 measured.
//   16 tb rows by 16 r of the matrix a workgroup: 2.5 a call, and a round of workgroups 0.12, 0.2, 0.37, 0.55 a block of columns for tb = 1..4 (0.3, 0.6
//     for 1, 2): 16 rows by 4096 x 4096 6.8, 64 rows 20; by 16 384 x 4096 24, 128 rows 43;
//   128 rows by 128: 8 (what is summed first, and the beginning), 1.25 a block (3.6), 2.3 where two workgroups share a CU: 128 rows by 4096 x 4096 44,
//     1024 51, 2048 80; fp32 128 rows 135, 2048 202 (a tile of 65 to 96 rows 0.8 of it);
//   columns in parts: the parts' sums written and added, 2.5 and 8 bytes a sum and part at 4 TB/s: 40 rows by 8192 columns in one part 26, in four 15.
Plan plan_of(const bifeat_linear_spec *s, int64_t rows, int32_t dtype) {
    const bool wide = dtype == BIFEAT_F32;
    const int64_t rows16 = (s->out_features + 15) / 16, blocks = (s->in_features + 127) / 128;
    Plan best{};
    double least = 0.0;
    const auto consider = [&](Plan p, int64_t workgroups, double begin, double block, int64_t at_once, int64_t least_blocks) {
        for (p.split = 1; p.split <= 16 && (p.split == 1 || blocks / p.split >= least_blocks); p.split *= 2) {
            const double rounds = std::max(1.0, at_once == 256 ? (double)((workgroups * p.split + 255) / 256) : 0.92 * (double)(workgroups * p.split) / 256);
            const double us = begin + rounds * block * (double)((blocks + p.split - 1) / p.split) +
                              (p.split > 1 ? 2.5 + 8e-6 / 4 * (double)p.split * (double)rows * s->out_features : 0.0);
            if (best.split == 0 || us < least) best = p, least = us;
        }
    };
    const int tb = rows <= 16 ? 1 : rows <= 32 || wide ? 2 : rows <= 48 ? 3 : 4;
    // (one row by 8192 x 28 672: 31.5 us with r = 2, 29.2 with 4; by 4096 x 4096 4.9 with 1, 5.7 with 2, 7.7 with 4)
    const int r = tb > 1 ? (wide ? 2 : 4) : rows16 >= 1536 ? 4 : rows16 >= 512 ? 2 : 1;
    const double few[2][5] = {{0, 0.12, 0.2, 0.37, 0.55}, {0, 0.3, 0.6, 0, 0}};
    consider({false, tb, r, 1}, (rows16 + r - 1) / r * ((rows + 16 * tb - 1) / (16 * tb)), 2.5, few[wide][tb], 256, 8);
    if (rows > 64 && s->in_features >= 8) consider({true, 0, 0, 1}, (rows16 + 7) / 8 * ((rows + 127) / 128), 8.0, wide ? 3.6 : 1.25, 512, 4);
    return best;
}

bool rows_ok(const bifeat_linear_spec *s, const bifeat_expert_rows *r) {
    return r && r->tokens >= 0 && r->choices >= 1 && r->choices <= 64 && r->token_stride >= 0 && r->choice_stride >= 0 &&
           r->tokens <= (1 << 30) / r->choices;
}

// The memory of bifeat_linear_experts: the number of tiles, the tiles, the pairs in order, the parts' counts, the sums of x, 32-bit products.
struct Room {
    int tile;
    int64_t most_tiles, order, counts, sums, products, bytes;
    int64_t sum_rows;  // of many rows: rows of x
};
Room room_of(const bifeat_linear_spec *s, const bifeat_expert_rows *r) {
    Room o;
    const int64_t pairs = r->tokens * r->choices;
    // Tiles of up to 128 pairs where an expert has 16 on the average, and where so large ones are enough for the whole card: there 14 000 pairs times 128-row
    // tiles of the matrix.  In tiles of 16 and of 128, of 16 bits: 64 matrices of 1536 x 2048 with 16 pairs each 37 us and 38, with 32 57 and 45, with 48 77 and 61; 128
    // of 2048 x 768 with 16 44 and 42, with 32 71 and 52; 16 of 4096 x 4096 with 16 41 and 36, with 24 51 and 47; 200 of 512 x 1024 with 16 27 and 30, with 32 40 and 38;
    // 8 of 1024 x 1024 with 96 15 and 22; 32 of them with 48 21 and 23, with 96 33 and 31; 8 of 4096 x 4096 with 24 31 and 36, with 48 47 and 44.  Rows of 32 bits pass
    // over at the same numbers, though their 128 cost more: the first with 16 75 and 86, with 24 97 and 97, with 48 162 and 142; the second with 16 83 and 84, with 32 135
    // and 104; 200 of 512 x 1024 with 24 63 and 62; 32 of 1024 x 1024 with 48 38 and 46, with 96 63 and 61; 8 of 4096 x 4096 with 48 98 and 123, with 96 179 and 162.
    // (By the average: where pairs are is not known here, so that few pairs that crowd on few experts are taken by 16.)
    o.tile = pairs >= 16 * (int64_t)s->experts && pairs * ((s->out_features + 127) / 128) >= 14000 && s->in_features >= 8 ? bf::kManyRows : 16;
    o.most_tiles = pairs / o.tile + std::min<int64_t>(pairs, s->experts + 1);
    o.order = 16 + (o.most_tiles + 1) / 2 * 16;  // (a tile is 8 bytes)
    static_assert(sizeof(bf::Tile) == 8, "");
    o.counts = o.order + o.most_tiles * o.tile * 4;
    const int parts = bf::deal_parts(pairs);
    o.sums = o.counts + (parts > 1 ? ((int64_t)parts * (s->experts + 1) + 3) / 4 * 16 : 0);
    o.sum_rows = o.tile == 16 ? 0 : r->choice_stride ? pairs : r->tokens;
    o.products = o.sums + sum_bytes(s, o.sum_rows);
    o.bytes = o.products + (r->weights ? pairs * s->out_features * 4 : 0);
    return o;
}

// Whether one of `rows` rows, `stride` elements apart, and `bytes` of out share memory.
bool meets(const void *x, int64_t rows, int64_t stride, int64_t columns, int32_t dtype, const void *out, int64_t bytes) {
    const __int128 element = dtype == BIFEAT_F32 ? 4 : 2, apart = stride * element, row = columns * element;
    const __int128 begin = (__int128)(uintptr_t)out - (__int128)(uintptr_t)x, end = begin + bytes;
    // (the first row that ends behind out's beginning)
    const __int128 first = row > begin ? 0 : apart == 0 ? rows : (begin - row) / apart + 1;
    return first < rows && first * apart < end;
}

}  // namespace

extern "C" {

int64_t bifeat_linear_bytes(const bifeat_linear_spec *spec) { return spec_ok(spec) ? matrices_of(spec, nullptr).bytes : BIFEAT_EINVAL; }

int bifeat_linear_pack(const bifeat_linear_spec *spec, const void *weight, int32_t dtype, uint8_t *packed, void *stream) {
    if (!spec_ok(spec) || !type_ok(dtype) || !data_ok(weight, dtype) || !packed || (uintptr_t)packed % 16) return BIFEAT_EINVAL;
    BF_HIP(bf::launch_linear_pack(matrices_of(spec, packed), spec->group, weight, dtype, packed, (hipStream_t)stream));
    return BIFEAT_OK;
}

int bifeat_linear_unpack(const bifeat_linear_spec *spec, const uint8_t *packed, float *weight, void *stream) {
    if (!spec_ok(spec) || !data_ok(weight, BIFEAT_F32) || !packed || (uintptr_t)packed % 16) return BIFEAT_EINVAL;
    BF_HIP(bf::launch_linear_unpack(matrices_of(spec, packed), spec->group, weight, (hipStream_t)stream));
    return BIFEAT_OK;
}

int64_t bifeat_linear_workspace(const bifeat_linear_spec *spec, int64_t rows, int32_t dtype) {
    if (!spec_ok(spec) || spec->experts != 1 || !type_ok(dtype) || rows < 0 || rows > INT32_MAX - 64) return BIFEAT_EINVAL;
    return plan_of(spec, rows, dtype).bytes(spec, rows);
}

int bifeat_linear_multiply(const bifeat_linear_spec *spec, const uint8_t *packed, const void *x, int64_t row_stride, int64_t rows,
                           int32_t dtype, void *out, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!spec_ok(spec) || spec->experts != 1 || !type_ok(dtype) || rows < 0 || rows > INT32_MAX - 64 || row_stride < 0) return BIFEAT_EINVAL;
    if (rows == 0) return BIFEAT_OK;
    if (!packed || (uintptr_t)packed % 16 || !data_ok(x, dtype) || !data_ok(out, dtype) || (uintptr_t)workspace % 16) return BIFEAT_EINVAL;
    // (others read x while out is written)
    if (meets(x, rows, row_stride, spec->in_features, dtype, out, rows * spec->out_features * (dtype == BIFEAT_F32 ? 4 : 2))) return BIFEAT_EINVAL;
    const Plan plan = plan_of(spec, rows, dtype);
    if (plan.bytes(spec, rows) > (workspace ? workspace_bytes : 0)) return BIFEAT_EINVAL;
    const bf::Matrices m = matrices_of(spec, packed);
    const hipStream_t s = (hipStream_t)stream;
    const bool split = plan.split > 1;
    bf::XRows r{x, row_stride, 0, 1, rows, split ? workspace : out, nullptr, rows};
    if (plan.many) {
        r.sums = reinterpret_cast<const uint2 *>(static_cast<uint8_t *>(workspace) + plan.parts_bytes(spec, rows));
        BF_HIP(bf::launch_linear_sums(m, spec->group, r, dtype, s));
        BF_HIP(bf::launch_linear_many(m, spec->group, r, nullptr, 0, dtype, split, plan.split, s));
    } else BF_HIP(bf::launch_linear_few(m, spec->group, r, nullptr, 0, dtype, split, {plan.tb, plan.r, plan.split, 8}, s));
    if (split) BF_HIP(bf::launch_linear_add(static_cast<const float *>(workspace), plan.split, rows * m.N, dtype, out, s));
    return BIFEAT_OK;
}

int64_t bifeat_linear_experts_workspace(const bifeat_linear_spec *spec, const bifeat_expert_rows *rows) {
    return spec_ok(spec) && rows_ok(spec, rows) ? room_of(spec, rows).bytes : (int64_t)BIFEAT_EINVAL;
}

int bifeat_linear_experts(const bifeat_linear_spec *spec, const uint8_t *packed, const bifeat_expert_rows *r, int32_t dtype, void *out,
                          void *workspace, int64_t workspace_bytes, void *stream) {
    if (!spec_ok(spec) || !type_ok(dtype) || !rows_ok(spec, r)) return BIFEAT_EINVAL;
    if (r->tokens == 0) return BIFEAT_OK;
    if (!packed || (uintptr_t)packed % 16 || !data_ok(r->x, dtype) || !data_ok(out, dtype) || !r->ids || (uintptr_t)r->ids % 4 ||
        (uintptr_t)r->weights % 4 || !workspace || (uintptr_t)workspace % 16)
        return BIFEAT_EINVAL;
    const int64_t outputs = r->tokens * (r->weights ? 1 : r->choices) * spec->out_features;
    for (int j = 0; j < (r->choice_stride ? r->choices : 1); j++) {
        const uint8_t *x = static_cast<const uint8_t *>(r->x);
        const int64_t element = dtype == BIFEAT_F32 ? 4 : 2;
        if (meets(x + j * r->choice_stride * element, r->tokens, r->token_stride, spec->in_features, dtype, out, outputs * element)) return BIFEAT_EINVAL;
    }
    const Room room = room_of(spec, r);
    if (workspace_bytes < room.bytes) return BIFEAT_EINVAL;
    const bf::Matrices m = matrices_of(spec, packed);
    const hipStream_t s = (hipStream_t)stream;
    const int64_t pairs = r->tokens * r->choices;
    uint8_t *w = static_cast<uint8_t *>(workspace);
    int *tiles_count = reinterpret_cast<int *>(w), *order = reinterpret_cast<int *>(w + room.order);
    bf::Tile *tiles = reinterpret_cast<bf::Tile *>(w + 16);
    float *products = reinterpret_cast<float *>(w + room.products);
    BF_HIP(bf::launch_linear_deal(r->ids, (int)pairs, spec->experts, room.tile, reinterpret_cast<int *>(w + room.counts), tiles_count, tiles, order, s));
    const bf::Deal deal{tiles_count, tiles, order};
    const bf::XRows x{r->x, r->token_stride, r->choice_stride, r->choices, pairs, r->weights ? (void *)products : out,
                      reinterpret_cast<const uint2 *>(w + room.sums), room.sum_rows};
    const bool to_float = r->weights != nullptr;
    // many workgroups have four waves each: a wave then has more blocks to go through, and the beginnings and ends of the others beside it (32 tokens of 8
    // of 128 experts of 1536 x 2048 54 us by eight waves and 32 rows, 45 by four, 43 by four and 64 rows; one token 8.7 and 9.4)
    const int waves = room.most_tiles * m.rows >= 2048 ? 4 : 8;
    if (room.tile == 16) BF_HIP(bf::launch_linear_few(m, spec->group, x, &deal, (int)room.most_tiles, dtype, to_float, {1, waves == 4 ? 4 : 2, 1, waves}, s));
    else {
        BF_HIP(bf::launch_linear_sums(m, spec->group, x, dtype, s));
        BF_HIP(bf::launch_linear_many(m, spec->group, x, &deal, (int)room.most_tiles, dtype, to_float, 1, s));
    }
    if (r->weights) BF_HIP(bf::launch_linear_join(products, r->ids, r->weights, r->tokens, r->choices, spec->experts, m.N, dtype, out, s));
    return BIFEAT_OK;
}

}  // extern "C"
