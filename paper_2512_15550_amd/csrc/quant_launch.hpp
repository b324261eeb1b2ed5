// Attention over 8-bit rows: the choice of the kernel's form.  Compiled for each type of query by itself (quant_bf16.hip, quant_f32.hip).
#pragma once
#include "cache_host.hpp"
#include "rows.hpp"
#include "sight_plan.hpp"
#include "tokens.hpp"

namespace ctkvr {

template <typename T> int quant_attn_launch(const ctkvr_cache *c, QuantAttnArgs &q, const SightPlan &plan, int store, int sight, int opt, hipStream_t st);

#ifdef CTKVR_QUANT_TYPE
template <typename T, int STORE, int SIGHT> int quant_attn_form(QuantAttnArgs &q, int log, int opt, unsigned grid, hipStream_t st)
{
    return with_opts(SIGHT == kTree ? opt & kCap : opt, [&](auto o) {
        constexpr int kOpt = decltype(o)::value & (SIGHT == kTree ? kCap : ~0);   // (drafted tokens have no distance)
        constexpr bool kWide = sizeof(T) == 2;
        if (log == 4) tokens_kernel<STORE, T, kOpt, SIGHT, 1><<<dim3(grid), 256, 0, st>>>(q);
        else if (log == 7) rows_kernel<STORE, T, kOpt, SIGHT, 4><<<dim3(grid), 256, 0, st>>>(q);
        else if (!kWide || (log != 5 && log != 8)) return no_kernel(log);
        if constexpr (kWide) {
            if (log == 5) tokens_kernel<STORE, T, kOpt, SIGHT, 2><<<dim3(grid), 256, 0, st>>>(q);
            if (log == 8) rows_kernel<STORE, T, kOpt, SIGHT, 8><<<dim3(grid), 512, 0, st>>>(q);
        }
        return (int)CTKVR_OK;
    });
}
template <typename T> int quant_attn_launch(const ctkvr_cache *c, QuantAttnArgs &q, const SightPlan &plan, int store, int sight, int opt, hipStream_t st)
{
    AttnArgs &a = q.a;
    const unsigned grid = (unsigned)((int64_t)a.tiles * c->p.n_kv_heads * a.nsplit);
    auto form = [&](auto store_, auto sight_) {
        return quant_attn_form<T, decltype(store_)::value, decltype(sight_)::value>(q, plan.log, opt, grid, st);
    };
    auto with_sight = [&](auto store_) {
        if (sight == kRange) return form(store_, std::integral_constant<int, kRange>());
        if (sight == kWindow) return form(store_, std::integral_constant<int, kWindow>());
        return form(store_, std::integral_constant<int, kTree>());
    };
    TRY(store == kInt8 ? with_sight(std::integral_constant<int, kInt8>()) : with_sight(std::integral_constant<int, kFp8>()));
    join_launch<T>(c, a, st);
    return launched("attention over 8-bit rows");
}
template int quant_attn_launch<CTKVR_QUANT_TYPE>(const ctkvr_cache *, QuantAttnArgs &, const SightPlan &, int, int, int, hipStream_t);
#endif

}  // namespace ctkvr
