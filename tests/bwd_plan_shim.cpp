// C entries over csrc/attn_bwd_plan.h for tests/test_bwd_plan_cpu.py.
#include <algorithm>
#include <chrono>
#include <vector>

#include "../paper_2603_24517_amd/csrc/attn_bwd_plan.h"

using namespace attn_bwd_plan;

static int plan(const int *call, Plan &r)
{
    const int rc = check_sizes(call[0], call[1], call[2], call[3], call[4], HD);
    return rc == ATTN_OK ? make_plan(call[0], call[1], call[2], call[3], call[4], call[5], r) : rc;
}

// call: B, Hq, Hkv, Sq, Skv, causal.  out: groups (B * Hkv), groups of an XCD or 0, together; keys items: tiles, pieces, window, grid; rows items: the same; all
// bytes of the workspace.
extern "C" int plan_of(const int *call, long long *out)
{
    Plan r = {};
    const int rc = plan(call, r);
    if (rc != ATTN_OK) return rc;
    const Sizes &p = r.p;
    long long *at = out;
    *at++ = p.keys.groups; *at++ = p.xcd_groups; *at++ = p.together;
    for (const Role *x : {&p.keys, &p.rows}) {
        *at++ = x->tiles; *at++ = x->splits; *at++ = x->window; *at++ = x->items;
    }
    *at = (long long)r.total;
    return ATTN_OK;
}

// Seconds that the fastest of 5 plans takes.
extern "C" double plan_seconds(const int *call)
{
    double best = 1e9;
    for (int n = 0; n < 5; ++n) {
        Plan r = {};
        const auto t = std::chrono::steady_clock::now();
        plan(call, r);
        best = std::min(best, std::chrono::duration<double>(std::chrono::steady_clock::now() - t).count());
    }
    return best;
}

// Deals out all workgroups of a call.  0 if every piece of every tile comes once, on the XCD that its group belongs to, with an order of groups that is
// whole windows; the pieces of a tile are all of its steps; the wavefronts' rows are all rows of the call, each once; and no unmasked pair of row and key is
// in none of the steps.  Otherwise the number of what is wrong.
extern "C" int deal_check(const int *call)
{
    Plan r = {};
    if (plan(call, r) != ATTN_OK) return 1;
    const Sizes &p = r.p;
    for (const Role *x : {&p.keys, &p.rows})
        if ((long long)x->groups * x->tiles * x->splits != x->items || x->window < 1) return 2;
    std::vector<uint8_t> seen[2] = {std::vector<uint8_t>(p.rows.items), std::vector<uint8_t>(p.keys.items)};
    for (int n = 0; n < p.keys.items + p.rows.items; ++n) {
        const Item i = which_item(p, n);
        const Role &x = i.keys ? p.keys : p.rows;
        if (i.group < 0 || i.group >= x.groups || i.tile < 0 || i.tile >= x.tiles || i.piece < 0 || i.piece >= x.splits) return 3;
        if (seen[i.keys][((size_t)i.tile * x.groups + i.group) * x.splits + i.piece]++) return 4;
        if (p.xcd_groups && (i.keys ? i.group : i.group / p.chunks) / p.xcd_groups != n % 8) return 5;
    }
    for (const auto &s : seen)
        if (std::find(s.begin(), s.end(), 0) != s.end()) return 6;
    for (int keys = 0; keys < 2; ++keys) {
        const Role &x = keys ? p.keys : p.rows;
        const int heads = keys ? p.Hkv : p.Hq, held = keys ? p.Skv : p.Sq;
        std::vector<uint8_t> rows((size_t)p.B * heads * ((held + 31) / 32));
        for (int t = 0; t < x.tiles; ++t) {
            const int steps = keys ? keys_steps(p, t) : rows_steps(p, t), n = pieces(steps, x.most);
            if (n > x.splits || steps < 0 || (keys && steps == 0)) return 7;
            int next = 0;
            for (int i = 0; i < n; ++i) {
                int first = 0, count = steps;
                if (n > 1) piece_steps(steps, n, i, first, count);
                if (first != next || count < (steps > 0) || count > x.most) return 8;
                next += count;
            }
            if (next != steps) return 9;
            for (int g = 0; g < x.groups; ++g)
                for (int wave = 0; wave < 4; ++wave) {
                    int b, head, x0;
                    find_rows(p, keys, g, t, wave, b, head, x0);
                    if (b < 0 || b >= p.B || head < 0 || head >= heads || x0 % 32) return 10;
                    if (x0 < held && rows[((size_t)b * heads + head) * ((held + 31) / 32) + x0 / 32]++) return 11;
                }
            // the first key of a keys tile that is not streamed to must be beyond every row in front of the first streamed one, and so on
            const long long off = call[5] ? (long long)p.Skv - p.Sq : (1ll << 40);
            if (keys) {
                const long long last_row = (long long)keys_skip(p, t) * BT - 1;
                if (last_row >= 0 && (long long)t * ITEM_ROWS <= std::min(last_row, (long long)p.Sq - 1) + off) return 12;
            } else {
                const long long last_row = std::min((t + 1ll) * (ITEM_ROWS >> p.pack_log2), (long long)p.Sq) - 1, first_key = (long long)steps * BT;
                if (first_key < p.Skv && first_key <= last_row + off) return 13;
            }
        }
        if (std::find(rows.begin(), rows.end(), 0) != rows.end()) return 14;
    }
    return 0;
}

#ifdef PLAN_MAIN
#include <stdio.h>
int main()
{
    int call[6];
    while (scanf("%d %d %d %d %d %d", call, call + 1, call + 2, call + 3, call + 4, call + 5) == 6) {
        long long out[12] = {};
        printf("%d\n", plan_of(call, out));
    }
}
#endif
