// Attention of a step's new rows over a KV cache in 8 bits: softmax(q . k / sqrt(d)) over what a row sees, times v.
//
// Mathematics.  One pass over the cache with, per row, a reference m of the exponents, l = sum of p and o = sum of p v for p = 2^(score * log2(e) - m);
// when m moves, l and o are multiplied by 2^(old - new).  m is not the running maximum but follows it lazily (REF_BELOW, REF_MOST), so that hardly any block
// pays for it.  Sums over waves and segments are brought to one m at the end.
//
// Products are float16 matrix instructions (16 x 16 x 32) with 32-bit sums: an 8-bit code is a float16 exactly, in either format, at one conversion per two
// codes.  The other operand is rounded to 11 bits or, for float32 queries, split into hi + lo with 22: queries after their row's largest has been
// brought below 2^15 by a power of two, probabilities as they are.  K's scales join the factor of the exponent; V's go into the conversion of its codes, relative
// to the largest one so far, where float16 holds that (V_ABOVE, V_BELOW).
//
// Layout and split.  A score product gives a lane four positions of one query row, twice a block: just what the second product takes from it as an operand (V is
// stored for that), so probabilities stay in registers.  Queries lie in LDS as operands.  A workgroup is four or eight waves on the
// blocks of one (sequence, kv head) in turn; a wave requests a block's K and V as soon as it has used those before.  Sequences are cut into segments by the
// plan (kv8_plan, cut_of), joined inside the launch where one die can hold them.
//
// What bounds it: from some thousands of positions a chip's worth of workgroups on the stream of the cache.  us, captured (and called one behind the other, where
// launches overlap): 8B, B = 4, n = 9, 32768 bf16 269 MB in 58 (55), 4.6 TB/s, of which some 45 stream at 6 TB/s, as fast as the blocks are read in the same
// order by a kernel that does nothing else (46 us), around them 5 until K is there and the queries are operands and 3 for the sums of waves and segments;
// float32 queries 68 (twice the products).  B = 32, n = 5, 1024..4096 173 MB in 47 (42): one workgroup per head and sequence, so the longest decides; all
// of 2500 35.8.  Short ones on the chain of round trips: arguments, lens, page, block, sums of waves, partial results, their arrival: B = 1, n = 9, 2048
// float32 9.7 (8.9), of which K is requested after 2.2 and the rows are joined in the last 2.
#include "kv8_launch.h"

// How a call is cut, by what the host knows of it.  A pass over the cache takes one to three row tiles of queries; more tiles read the cache less often, but
// their workgroups have more to set up, to add over their waves and to join.
//  - Short sequences (as long as they can be: `blocks`): a tile a pass, while its workgroups fit on the chip together.  us, one tile / as few passes as
//    can be, of 9 rows of 8B: float32 B = 1, 300 8.2 / 11.4, 2048 9.2 / 11.5, 8192 13.9 / 16.2, 16384 18.8 / 19.3, 32768 29.0 / 26.6; B = 8, 2048
//    19.5 / 20.0, 4096 30.6 / 26.9; bf16 B = 1, 8192 13.5 / 14.8, 16384 18.2 / 17.2; two
//    tiles, n = 5, bf16 B = 5, 1000 10.1 / 10.4, 2048 13.3 / 12.1; 70B float32 B = 5, 300 7.4 / 13.5; B = 6, 1500 15.5 / 22.3; sixteen tiles, n = 32,
//    B = 3, 1000 16.6 / 21.6, B = 1, 4000 21.0 / 17.6, bf16 B = 2, 4000 25.9 / 20.9; more workgroups than fit, 8B B = 16, n = 32, 500 18.5 / 13.8.
//  - Else by rounds of 256 workgroups and what a block costs a pass of one, two and three tiles.  us, by that / fewest passes / one tile: 70B float32
//    B = 7, n = 13, 700..1500 21.4 / 26.8 / 21.0; B = 2, n = 32, 4000 bf16 20.9 / 24.9 / 25.8; 8B B = 16, n = 32, 500 13.8 / 16.9 / 18.5;
//    B = 4, n = 9, 32768 57.4 / 57.7 / 76.8.
//  - Segments of a sequence so that 256 workgroups have work; twice that where 256 in whole segments leave a quarter of the chip idle (8B B = 12, 3000
//    24.6, without 27.8; for all calls: B = 32, 2500 41, now 36).
// The limits were found with 8 kv heads of 128 channels; others go by the same ones, unmeasured.
Kv8Plan kv8_plan(int B, int n, int gq, int nkv, int blocks, bool f32)
{
    const int tiles = (n * gq + 15) / 16;
    const int64_t heads = (int64_t)B * nkv;
    Kv8Plan p;
    const bool brief = heads * blocks <= (f32 ? 3500 : tiles > 2 ? 2750 : 2000) && heads * blocks * tiles <= 15000 && heads * tiles <= 512;
    if (brief) p.passes = tiles;
    double best = 0;
    for (int rt = KV8_MAX_TILES; rt >= 1 && !brief; --rt) {
        const int passes = (tiles + rt - 1) / rt;
        const int64_t units = heads * passes;
        static const double block[4] = {0, 0.75, 1.0, 1.4};
        const double cost = units <= 256 ? block[rt] / (256 / units) : block[rt] * ((units + 255) / 256);
        if (rt == KV8_MAX_TILES || cost < best) {
            best = cost;
            p.passes = passes;
        }
    }
    const int64_t units = heads * p.passes;
    int64_t share = 256 / units;
    if (share * units <= 192) share = 512 / units;
    p.share = share < 1 ? 1 : share > 64 ? 64 : (int)share;
    p.in_die = heads % 8 == 0 && units <= HAND_GROUPS;
    return p;
}

size_t kv8_attention_ws(int d) { return HAND_WORDS + (size_t)KV8_GROUPS * KV8_MAX_TILES * 16 * (d * sizeof(float) + sizeof(f32x4)); }

hipError_t launch_kv8_attention(Kv8AttnArgs a, int fmt, int d, void *ws, hipStream_t s) { return launch_attention<KV8_ALONE>(a, fmt, d, ws, s); }
