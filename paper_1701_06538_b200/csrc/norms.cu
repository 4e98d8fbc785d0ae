// The norms around the block, one pass over memory each way.
//   norm_in:   xn = x r w,                              r  = (mean x^2 + eps)^-1/2
//   norm_out:  out = residual_scale x + gate (y r w),   r  = (mean y^2 + eps)^-1/2
//              next = out r2 w_next,                    r2 = (mean out^2 + eps)^-1/2   (the norm before the next block)
// Backward, with n = y r and n2 = out r2:
//   dt = dOut + r2 (dNext w_next - n2 mean(dNext w_next n2)),   dX = residual_scale dt,   dw_next = sum of dNext n2
//   dY = r (dt gate w - n mean(dt gate w n)),   dgate = w times the sum of dt n over the rows of the gate,   dw = sum of dt gate n
// All of it is bound by memory: a row stays in registers between its sums and what is made of it. Sums are float, over rows first by
// threads that keep their columns, then in double over what blocks have left, in a fixed order.
#include "async_copy.cuh"
#include "block.cuh"
#include "pairs.cuh"
#include "vectors.cuh"

namespace moe {

namespace {

// A row belongs to a team of `warps` warps of the block. Sums over the team's threads; `sh` has a place per warp and sum, twice, so that one
// barrier a row is enough: who writes the next row's sums does so on the other side, and the barrier of that row keeps it from coming round.
constexpr int MAX_SUMS = 4;
__device__ __forceinline__ void team_barrier(int warps, int team) { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(warps * 32) : "memory"); }
__device__ __forceinline__ float team_sum(float s, int warps, float *sh, int &side) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (warps == 1) return s;
    const int warp = threadIdx.x >> 5, team = warp / warps;
    float *mine = sh + side * (32 * MAX_SUMS);
    side ^= 1;
    if ((threadIdx.x & 31) == 0) mine[warp] = s;
    team_barrier(warps, team);
    s = 0.0f;
    for (int q = 0; q < warps; ++q) s += mine[team * warps + q];
    return s;
}
// Four at once: lanes give away half of their sums in the first two steps, so that six exchanges do instead of twenty. Lane l then has sum l / 8.
__device__ __forceinline__ void team_sums(float (&s)[4], int warps, float *sh, int &side) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, team = warp / warps;
    const bool hi = lane & 16, up = lane & 8;
    float a = hi ? s[2] : s[0], b = hi ? s[3] : s[1];
    a += __shfl_xor_sync(0xffffffffu, hi ? s[0] : s[2], 16);
    b += __shfl_xor_sync(0xffffffffu, hi ? s[1] : s[3], 16);
    float t = up ? b : a;
    t += __shfl_xor_sync(0xffffffffu, up ? a : b, 8);
#pragma unroll
    for (int off = 4; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
    if (warps == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = __shfl_sync(0xffffffffu, t, 8 * i);
        return;
    }
    float4 *mine = reinterpret_cast<float4 *>(sh + side * (32 * MAX_SUMS));
    side ^= 1;
    if ((lane & 7) == 0) reinterpret_cast<float *>(mine + warp)[lane >> 3] = t;
    team_barrier(warps, team);
    float4 all = mine[team * warps];
    for (int q = 1; q < warps; ++q) {
        const float4 f = mine[team * warps + q];
        all.x += f.x; all.y += f.y; all.z += f.z; all.w += f.w;
    }
    s[0] = all.x; s[1] = all.y; s[2] = all.z; s[3] = all.w;
}

// Y: the block's output goes through its norm and the gate onto x; NEXT: a norm of the result (without Y: of x). Arithmetic in pairs: element by element it was 31 instructions an element
// and kept memory waiting, 28.2 us for 32768 x 512. AHEAD: a team has several rows and the next one on its way; else one.
template <typename T, int V, bool Y, bool NEXT, bool GATE, bool AHEAD>
__global__ void __launch_bounds__(512) norm_rows_kernel(const NormArgs a, int warps) {
    wait_previous_kernel();
    constexpr int N = Vec<T>::N, P = N / 2;
    __shared__ float sh[2 * 32 * MAX_SUMS];
    int side = 0;
    const int threads = warps * 32, teams = blockDim.x / threads, lane = threadIdx.x % threads;
    const int64_t stride = (int64_t)gridDim.x * teams;
    const int32_t pieces = a.d / N;
    const float by = 1.0f / (float)a.d;
    struct Row { Vec<T> x[V], y[Y ? V : 1]; };
    auto fetch = [&](Row &f, int64_t row) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            if constexpr (Y) f.y[v] = load_vec<T>(a.y, row, a.d, q);
            f.x[v] = load_vec<T>(a.x, row, a.d, q);
        }
    };
    Row next;
    int64_t row = (int64_t)blockIdx.x * teams + threadIdx.x / threads;
    if (row < a.T) fetch(next, row);
#pragma unroll 1
    for (; row < a.T; row += AHEAD ? stride : a.T) {
        const Row now = next;
        if (AHEAD && row + stride < a.T) fetch(next, row + stride);
        float2 o[V][P];
        float2 sum = both(0.0f);
        if constexpr (Y) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (lane + v * threads < pieces)
#pragma unroll
                    for (int i = 0; i < P; ++i) { const float2 f = now.y[v].get(2 * i); sum = fma2(f, f, sum); }
            const float r = 1.0f / sqrtf(team_sum(sum.x + sum.y, warps, sh, side) * by + a.eps);
            if (lane == 0) a.rstd[row] = r;
            const int64_t gate_row = GATE ? (int64_t)((uint32_t)row / (uint32_t)a.rows_per_gate) : 0;
            sum = both(0.0f);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int32_t q = lane + v * threads;
                if (q >= pieces) break;
                float2 w[P];
                load_floats(a.w + (int64_t)q * N, w);
                Vec<T> g, res;
                if constexpr (GATE) g = load_vec<T>(a.gate, gate_row, a.d, q);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    float2 u = mul2(mul2(now.y[v].get(2 * i), both(r)), w[i]);
                    if constexpr (GATE) u = mul2(u, g.get(2 * i));
                    o[v][i] = fma2(both(a.residual_scale), now.x[v].get(2 * i), u);
                    sum = fma2(o[v][i], o[v][i], sum);
                    res.set(2 * i, o[v][i]);
                }
                store_vec<T>(a.out, row, a.d, q, res);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (lane + v * threads < pieces)
#pragma unroll
                    for (int i = 0; i < P; ++i) { o[v][i] = now.x[v].get(2 * i); sum = fma2(o[v][i], o[v][i], sum); }
        }
        if constexpr (NEXT) {  // of what was not rounded yet
            const float r = 1.0f / sqrtf(team_sum(sum.x + sum.y, warps, sh, side) * by + a.eps);
            if (lane == 0 && a.rstd_next) a.rstd_next[row] = r;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int32_t q = lane + v * threads;
                if (q >= pieces) break;
                float2 w[P];
                load_floats(a.w_next + (int64_t)q * N, w);
                Vec<T> res;
#pragma unroll
                for (int i = 0; i < P; ++i) res.set(2 * i, mul2(mul2(o[v][i], both(r)), w[i]));
                store_vec<T>(a.next, row, a.d, q, res);
            }
        }
    }
}

// How the backward pass shares out its rows. With one gate (or none) a block has `rows` rows of one group and leaves partial sums (chunks of a
// group: `chunks`); with groups of a few rows a team has whole groups and writes their gate's gradient itself (chunks 0).
struct Share {
    int warps, teams, V, ring;  // ring: rows that a warp holds in shared memory (0: a row of several warps, in registers)
    int64_t group, groups, chunks, rows, per_team, blocks, most;  // per_team: groups a team takes (chunks == 0); most: blocks that the workspace has room for
};
constexpr int TEAM_ROWS = 4;  // 8192 x 512, main and sums: 10.3 us; 1, 2 and 3 rows 14.2, 14.5 and 11.9
// rows of a team when blocks are two waves of one an SM (where blocks are large) or of three: what the workspace has room for goes by it
int64_t team_rows(int64_t T, int teams) { return imax(TEAM_ROWS, cdiv(T, (int64_t)teams * 148 * (teams > 8 ? 2 : 6))); }
// Forward: a warp has a row up to 32 vectors a lane, else several do
void team_of(int32_t d, int32_t act, int *warps, int *teams, int *V) {
    const int64_t pieces = d / (16 / (int64_t)act_bytes(act));
    *V = pieces <= 32 ? 1 : pieces <= 1024 ? 2 : pieces <= 2048 ? 4 : 8;  // at most 512 threads
    int w = 1;
    while (w * 32 * *V < pieces) w *= 2;
    *warps = w;
    *teams = w >= 8 ? 1 : 8 / w;
}
// Backward: a warp has a row of up to 128 vectors, and the next one on its way to shared memory; wider rows are a vector a thread while 512 threads do
constexpr int STREAM_PIECES = 128, RING_ROWS = 2, SHARED_MOST = 200 * 1024, SHARED_ALLOWED = 216 * 1024;  // beside the rings: w and w_next, 8 KiB at most
// warps of a block: eight where three blocks or two have room, else as many as one has
int64_t stream_warps(int64_t row) { return row * 8 <= SHARED_MOST / 2 ? 8 : imin(12, SHARED_MOST / row); }
void grad_team_of(int32_t d, int32_t act, int tensors, int *warps, int *teams, int *V, int *ring) {
    const int64_t pieces = d / (16 / (int64_t)act_bytes(act));
    if (pieces <= STREAM_PIECES) {
        const int64_t row = (int64_t)tensors * d * (int64_t)act_bytes(act) * RING_ROWS;
        *V = pieces <= 32 ? 1 : pieces <= 64 ? 2 : 4;
        *warps = 1;
        *ring = RING_ROWS;
        *teams = (int)stream_warps(row);
        return;
    }
    *ring = 0;
    *V = pieces <= 512 ? 1 : pieces <= 1024 ? 2 : pieces <= 2048 ? 4 : 8;
    *warps = (int)cdiv(pieces, 32 * *V);  // at least five
    *teams = 1;
}
// more blocks than share_of() takes: whole groups fill at least half of a block's rows, and beside the chunks of `rows` rows there is at most one
// that is not full for every group, of more than 3 * each rows
int64_t most_blocks(int64_t T, int teams) {
    const int64_t each = team_rows(T, teams);
    return 2 * cdiv(T, each * teams) + T / (3 * each) + 3;
}
// Blocks all have the same work and run in waves of as many as the SMs hold (two each where three have room: the third gains less than its start costs); each costs START rows' time
// before and behind its rows. Of the shares of one wave to sixteen, and of whole groups to three quarters of the teams, the one that takes least. 131072 x 1024:
// with a gate for 64 rows 342 us, 520 where 1.2 waves of blocks had them; for 512 rows 295, 373 in chunks of 444 and 68 rows; for 200 rows 300, 482 with five teams a block.
constexpr int64_t START = 16;
Share share_of(int64_t T, int32_t d, int32_t act, int tensors, int64_t rows_per_gate) {
    Share chunks = {}, whole = {};
    grad_team_of(d, act, tensors, &chunks.warps, &chunks.teams, &chunks.V, &chunks.ring);
    grad_team_of(d, act, tensors + 1, &whole.warps, &whole.teams, &whole.V, &whole.ring);  // their gates go through the ring too
    chunks.most = most_blocks(T, chunks.teams);
    whole.most = most_blocks(T, whole.teams);
    chunks.group = whole.group = rows_per_gate > 0 ? imin(rows_per_gate, imax(T, 1)) : imax(T, 1);
    chunks.groups = whole.groups = cdiv(T, chunks.group);
    const int64_t at_once = 148 * (chunks.teams > 8 ? 1 : 2), whole_at_once = 148 * (whole.teams > 8 ? 1 : 2);
    const int teams = whole.teams;
    int64_t best = INT64_MAX, best_whole = INT64_MAX;
    for (int64_t waves = 1; waves <= 16; ++waves) {
        Share s = chunks;
        const int64_t rows = cdiv(s.group, imax(1, waves * at_once / imax(1, s.groups)));
        s.rows = imin(s.group, imax(cdiv(rows, s.teams), TEAM_ROWS) * s.teams);
        s.chunks = cdiv(s.group, s.rows);
        s.blocks = s.groups * s.chunks;
        const int64_t cost = cdiv(s.blocks, at_once) * (s.rows + START);
        if (cost < best && s.blocks <= s.most) {
            best = cost;
            chunks = s;
        }
        if (rows_per_gate <= 0) continue;
        for (int t = teams; 4 * t >= 3 * teams; --t) {
            Share u = whole;
            u.teams = t;
            u.per_team = imax(imax(1, TEAM_ROWS / u.group), cdiv(u.groups, waves * whole_at_once * t));
            u.blocks = cdiv(u.groups, u.per_team * t);
            const int64_t of = cdiv(u.blocks, whole_at_once) * (t * u.per_team * u.group + START);
            if (of < best_whole && u.blocks <= u.most) {
                best_whole = of;
                whole = u;
            }
        }
    }
    return rows_per_gate > 0 && best_whole <= best ? whole : chunks;
}

// GATE: 0 none, 1 a block's rows have one, 2 groups of a few rows (chunks 0)
template <typename T, int V, bool Y, bool NEXT, int GATE>
__global__ void __maxnreg__(128) norm_grads_kernel(const NormGradArgs a, const Share s, float *part_w, float *part_next, float *part_gate) {
    wait_previous_kernel();
    constexpr int N = Vec<T>::N, P = N / 2;
    __shared__ __align__(16) float sh[2 * 32 * MAX_SUMS];
    int side = 0;
    const int threads = s.warps * 32, lane = threadIdx.x;  // one team
    const int32_t pieces = a.d / N;
    const float by = 1.0f / (float)a.d;
    float2 sum_n[Y ? V : 1][P], sum_w[GATE == 2 ? V : 1][P], sum_next[NEXT ? V : 1][P];  // of dt n over the group's rows so far; of dt gate n; of dNext n2
    float2 gw[Y ? V : 1][P], wn[NEXT ? V : 1][P];                                           // gate times w of the group (GATE 2: w); w_next
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int32_t q = lane + v * threads;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if constexpr (Y) sum_n[v][i] = both(0.0f);
            if constexpr (GATE == 2) sum_w[v][i] = both(0.0f);
            if constexpr (NEXT) sum_next[v][i] = both(0.0f);
        }
        if (q >= pieces) continue;
        if constexpr (Y && GATE != 1) load_floats(a.w + (int64_t)q * N, gw[v]);
        if constexpr (NEXT) load_floats(a.w_next + (int64_t)q * N, wn[v]);
    }
    auto begin_group = [&](int64_t gate_row) {
        if (GATE == 1)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int32_t q = lane + v * threads;
                if (q >= pieces) break;
                load_floats(a.w + (int64_t)q * N, gw[v]);
                const Vec<T> g = load_vec<T>(a.gate, gate_row, a.d, q);
#pragma unroll
                for (int i = 0; i < P; ++i) gw[v][i] = mul2(gw[v][i], g.get(2 * i));
            }
    };
    struct Row { Vec<T> dout[V], dnext[NEXT ? V : 1], out[NEXT ? V : 1], y[Y ? V : 1], gate[GATE == 2 ? V : 1]; float r, r2; };
    auto fetch = [&](Row &f, int64_t row, int64_t gate_row) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            if (a.dOut) f.dout[v] = load_vec<T>(a.dOut, row, a.d, q);
            else f.dout[v].raw = make_uint4(0u, 0u, 0u, 0u);
            if constexpr (NEXT) {
                f.dnext[v] = load_vec<T>(a.dNext, row, a.d, q);
                f.out[v] = load_vec<T>(a.out, row, a.d, q);
            }
            if constexpr (Y) f.y[v] = load_vec<T>(a.y, row, a.d, q);
            if constexpr (GATE == 2) f.gate[v] = load_vec<T>(a.gate, gate_row, a.d, q);
        }
        if constexpr (Y) f.r = a.rstd[row];
        if constexpr (NEXT) f.r2 = a.rstd_next[row];
    };
    auto one_row = [&](const Row &f, int64_t row) {
        auto gated = [&](int v, int i) {
            float2 w = gw[Y ? v : 0][i];
            if constexpr (GATE == 2) w = mul2(w, f.gate[v].get(2 * i));
            return w;
        };
        // c2 = mean(dn2 n2) decides dt, and c1 = mean(dt b) with b = gate w n the rest. Both are sums of one look at the row, since c1 is linear in dt:
        // mean(dOut b) + r2 (mean(dn2 b) - c2 mean(n2 b))
        float2 s0 = both(0.0f), s1 = s0, s2 = s0, s3 = s0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (lane + v * threads >= pieces) break;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float2 b;
                if constexpr (Y) {
                    b = mul2(mul2(f.y[v].get(2 * i), both(f.r)), gated(v, i));
                    s1 = fma2(f.dout[v].get(2 * i), b, s1);
                }
                if constexpr (NEXT) {
                    const float2 n2 = mul2(f.out[v].get(2 * i), both(f.r2)), dn2 = mul2(f.dnext[v].get(2 * i), wn[v][i]);
                    s0 = fma2(dn2, n2, s0);
                    if constexpr (Y) {
                        s2 = fma2(dn2, b, s2);
                        s3 = fma2(n2, b, s3);
                    }
                }
            }
        }
        float c1 = 0.0f, c2 = 0.0f;
        if constexpr (Y && NEXT) {
            float sum[4] = {s0.x + s0.y, s1.x + s1.y, s2.x + s2.y, s3.x + s3.y};
            team_sums(sum, s.warps, sh, side);
            c2 = sum[0] * by;
            c1 = (sum[1] + f.r2 * (sum[2] - c2 * sum[3])) * by;
        } else if constexpr (Y) {
            c1 = team_sum(s1.x + s1.y, s.warps, sh, side) * by;
        } else {
            c2 = team_sum(s0.x + s0.y, s.warps, sh, side) * by;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            Vec<T> dx, dy;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float2 dt = f.dout[v].get(2 * i);
                if constexpr (NEXT) {
                    const float2 n2 = mul2(f.out[v].get(2 * i), both(f.r2)), g2 = f.dnext[v].get(2 * i);
                    dt = fma2(both(f.r2), fma2(n2, both(-c2), mul2(g2, wn[v][i])), dt);
                    sum_next[v][i] = fma2(g2, n2, sum_next[v][i]);
                }
                dx.set(2 * i, mul2(both(a.residual_scale), dt));
                if constexpr (Y) {
                    const float2 n = mul2(f.y[v].get(2 * i), both(f.r));
                    dy.set(2 * i, mul2(both(f.r), fma2(n, both(-c1), mul2(dt, gated(v, i)))));
                    sum_n[v][i] = fma2(dt, n, sum_n[v][i]);
                }
            }
            store_vec<T>(a.dX, row, a.d, q, dx);
            if constexpr (Y) store_vec<T>(a.dY, row, a.d, q, dy);
        }
    };
    // rows one behind the other; GATE 2: from group to group, each with its end. With a vector a thread the next row is on its way meanwhile (32768 x 2048: 150 us, 199 without; with two
    // it is more than the registers hold: 8192 x 8192 190 without, 290 with it)
    auto some_rows = [&](int64_t row, int64_t end, int64_t g) {
        int64_t group_end = row + s.group;
        Row now;
        if (V == 1 && row < end) fetch(now, row, g);
#pragma unroll 1
        for (; row < end; ++row) {
            const bool ends = GATE == 2 && (row + 1 == group_end || row + 1 == end);
            Row next;
            if constexpr (V == 1) {
                next = now;
                if (row + 1 < end) fetch(next, row + 1, ends ? g + 1 : g);
            } else {
                fetch(now, row, g);
            }
            one_row(now, row);
            if (ends) {
#pragma unroll
                for (int v = 0; v < V; ++v) {  // the group's gate gradient, and its part of dw
                    const int32_t q = lane + v * threads;
                    if (q >= pieces) break;
                    Vec<T> dg;
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        float2 &n = sum_n[Y ? v : 0][i], &w = sum_w[GATE == 2 ? v : 0][i];
                        w = fma2(now.gate[GATE == 2 ? v : 0].get(2 * i), n, w);
                        dg.set(2 * i, mul2(gw[Y ? v : 0][i], n));
                        n = both(0.0f);
                    }
                    store_vec<T>(a.dgate, g, a.d, q, dg);
                }
                ++g;
                group_end += s.group;
            }
            if constexpr (V == 1) now = next;
        }
    };
    // done(vector of columns, their sums)
    auto block_sums = [&](auto &mine, auto done) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + v * threads;
            if (q >= pieces) break;
            done(q, mine[v]);
        }
    };
    auto to_part = [&](float *part) {
        return [=](int32_t q, const float2 (&total)[P]) {
#pragma unroll
            for (int i = 0; i < P; i += 2)
                *reinterpret_cast<float4 *>(part + (int64_t)blockIdx.x * a.d + (int64_t)q * N + 2 * i) = make_float4(total[i].x, total[i].y, total[i + 1].x, total[i + 1].y);
        };
    };

    if constexpr (GATE == 2) {
        const int64_t first = (int64_t)blockIdx.x * s.per_team;
        some_rows(first * s.group, min((first + s.per_team) * s.group, a.T), first);
        block_sums(sum_w, to_part(part_w));
    } else {
        const int64_t g = blockIdx.x / s.chunks, from = g * s.group + (blockIdx.x % s.chunks) * s.rows;
        begin_group(g);
        some_rows(from, min(min(from + s.rows, (g + 1) * s.group), a.T), g);
        if constexpr (GATE == 1) {
            block_sums(sum_n, [&](int32_t q, const float2 (&total)[P]) {
                const Vec<T> gv = load_vec<T>(a.gate, g, a.d, q);
                float2 w[P], of_w[P];
                load_floats(a.w + (int64_t)q * N, w);
                Vec<T> dg;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    of_w[i] = mul2(gv.get(2 * i), total[i]);
                    dg.set(2 * i, mul2(w[i], total[i]));
                }
                to_part(part_w)(q, of_w);
                if (s.chunks > 1) to_part(part_gate)(q, total);
                else store_vec<T>(a.dgate, g, a.d, q, dg);
            });
        } else if constexpr (Y) {
            block_sums(sum_n, to_part(part_w));
        }
    }
    if constexpr (NEXT) block_sums(sum_next, to_part(part_next));
}

// The same where a warp has a row: rows come by asynchronous copies, each lane's own pieces two rows ahead, into the warp's ring, so that registers hold nothing but the columns' sums and
// memory is kept busy whatever the warp is doing. (Rows in registers, four warps to a row of 1024: 331 us for 131072 rows, five tensors of whose bytes take 246.) w and w_next lie in shared
// memory, with the gate in w where the block has one.
template <typename T, int V, bool Y, bool NEXT, int GATE>
__global__ void __launch_bounds__(384) norm_stream_kernel(const NormGradArgs a, const Share s, float *part_w, float *part_next, float *part_gate) {
    wait_previous_kernel();
    constexpr int N = Vec<T>::N, P = N / 2, TENSORS = (Y ? 2 : 1) + (NEXT ? 2 : 0), HELD = TENSORS + (GATE == 2 ? 1 : 0);  // HELD: of a row in the ring; GATE 2: its gate is the last
    extern __shared__ __align__(16) char norm_shared[];
    const int32_t d = a.d, pieces = d / N;
    float *gw = reinterpret_cast<float *>(norm_shared), *wn = gw + (Y ? d : 0);
    uint4 *ring = reinterpret_cast<uint4 *>(wn + (NEXT ? d : 0));  // [warp][row][HELD][pieces]
    float *columns = reinterpret_cast<float *>(ring);             // afterwards: [warp][d]
    const int team = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint4 *mine = ring + (int64_t)team * RING_ROWS * HELD * pieces;
    const float by = 1.0f / (float)d;
    const int64_t block_group = GATE == 2 ? 0 : blockIdx.x / s.chunks;
    // a row's pieces of this lane, to place `at` of the ring; its factors go with it
    auto ask = [&](int64_t row, int64_t end, int at, int64_t gate_row) {
        if (row < end)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int32_t q = lane + 32 * v;
                if (q >= pieces) break;
                uint4 *to = mine + at * HELD * pieces + q;
                const int64_t from = row * d + (int64_t)q * N;
                if (a.dOut) copy16(to, static_cast<const T *>(a.dOut) + from);
                else zero16(to);
                if (Y) copy16(to + pieces, static_cast<const T *>(a.y) + from);
                if (NEXT) {
                    copy16(to + (Y ? 2 : 1) * pieces, static_cast<const T *>(a.dNext) + from);
                    copy16(to + (Y ? 3 : 2) * pieces, static_cast<const T *>(a.out) + from);
                }
                if (GATE == 2) copy16(to + TENSORS * pieces, static_cast<const T *>(a.gate) + gate_row * d + (int64_t)q * N);
            }
        copies_commit();
    };
    // the block's rows of this warp, or (GATE 2) its groups; the first row is on its way before everything else
    const int64_t first_group = ((int64_t)blockIdx.x * s.teams + team) * s.per_team;
    const int64_t first = GATE == 2 ? first_group * s.group : block_group * s.group + (blockIdx.x % s.chunks) * s.rows + team;
    const int64_t last = GATE == 2 ? min((first_group + s.per_team) * s.group, a.T) : min(min(first - team + s.rows, (block_group + 1) * s.group), a.T);
    ask(first, last, 0, first_group);
    for (int32_t q = threadIdx.x; q < pieces; q += blockDim.x) {
        float2 f[P];
        Vec<T> g;
        if constexpr (GATE == 1) g = load_vec<T>(a.gate, block_group, d, q);
        if constexpr (Y) {
            load_floats(a.w + (int64_t)q * N, f);
#pragma unroll
            for (int i = 0; i < P; ++i) *reinterpret_cast<float2 *>(gw + q * N + 2 * i) = GATE == 1 ? mul2(f[i], g.get(2 * i)) : f[i];
        }
        if constexpr (NEXT) {
            load_floats(a.w_next + (int64_t)q * N, f);
#pragma unroll
            for (int i = 0; i < P; ++i) *reinterpret_cast<float2 *>(wn + q * N + 2 * i) = f[i];
        }
    }
    __syncthreads();
    float2 sum_n[Y ? V : 1][P], sum_w[GATE == 2 ? V : 1][P], sum_next[NEXT ? V : 1][P];  // of dt n over the group's rows so far; of dt gate n; of dNext n2
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (Y) sum_n[Y ? v : 0][i] = both(0.0f);
            if (GATE == 2) sum_w[GATE == 2 ? v : 0][i] = both(0.0f);
            if (NEXT) sum_next[NEXT ? v : 0][i] = both(0.0f);
        }
    auto one_row = [&](int64_t row, int at) {
        const uint4 *held = mine + at * HELD * pieces;
        const float r = Y ? a.rstd[row] : 0.0f, r2 = NEXT ? a.rstd_next[row] : 0.0f;
        auto weights = [&](const float *from, int32_t q, float2 (&f)[P]) {
#pragma unroll
            for (int i = 0; i < P; i += 2) {
                const float4 x = *reinterpret_cast<const float4 *>(from + q * N + 2 * i);
                f[i] = make_float2(x.x, x.y);
                f[i + 1] = make_float2(x.z, x.w);
            }
        };
        auto gated = [&](int32_t q, float2 (&f)[P]) {
            weights(gw, q, f);
            if (GATE == 2) {
                Vec<T> g;
                g.raw = held[TENSORS * pieces + q];
#pragma unroll
                for (int i = 0; i < P; ++i) f[i] = mul2(f[i], g.get(2 * i));
            }
        };
        float2 s0 = both(0.0f), s1 = s0, s2 = s0, s3 = s0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + 32 * v;
            if (q >= pieces) break;
            Vec<T> dout, y, dnext, out;
            float2 b[P], f[P];
            dout.raw = held[q];
            if (Y) {
                y.raw = held[pieces + q];
                gated(q, b);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    b[i] = mul2(mul2(y.get(2 * i), both(r)), b[i]);
                    s1 = fma2(dout.get(2 * i), b[i], s1);
                }
            }
            if (NEXT) {
                dnext.raw = held[(Y ? 2 : 1) * pieces + q];
                out.raw = held[(Y ? 3 : 2) * pieces + q];
                weights(wn, q, f);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 n2 = mul2(out.get(2 * i), both(r2)), dn2 = mul2(dnext.get(2 * i), f[i]);
                    s0 = fma2(dn2, n2, s0);
                    if (Y) {
                        s2 = fma2(dn2, b[i], s2);
                        s3 = fma2(n2, b[i], s3);
                    }
                }
            }
        }
        float c1 = 0.0f, c2 = 0.0f;  // see norm_grads_kernel
        int side = 0;
        if (Y && NEXT) {
            float sum[4] = {s0.x + s0.y, s1.x + s1.y, s2.x + s2.y, s3.x + s3.y};
            team_sums(sum, 1, nullptr, side);
            c2 = sum[0] * by;
            c1 = (sum[1] + r2 * (sum[2] - c2 * sum[3])) * by;
        } else if (Y) {
            c1 = team_sum(s1.x + s1.y, 1, nullptr, side) * by;
        } else {
            c2 = team_sum(s0.x + s0.y, 1, nullptr, side) * by;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + 32 * v;
            if (q >= pieces) break;
            Vec<T> dout, y, dnext, out, dx, dy;
            float2 b[P], f[P];
            dout.raw = held[q];
            if (Y) {
                y.raw = held[pieces + q];
                gated(q, b);
            }
            if (NEXT) {
                dnext.raw = held[(Y ? 2 : 1) * pieces + q];
                out.raw = held[(Y ? 3 : 2) * pieces + q];
                weights(wn, q, f);
            }
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float2 dt = dout.get(2 * i);
                if (NEXT) {
                    const float2 n2 = mul2(out.get(2 * i), both(r2)), g2 = dnext.get(2 * i);
                    dt = fma2(both(r2), fma2(n2, both(-c2), mul2(g2, f[i])), dt);
                    float2 &sum = sum_next[NEXT ? v : 0][i];
                    sum = fma2(g2, n2, sum);
                }
                dx.set(2 * i, mul2(both(a.residual_scale), dt));
                if (Y) {
                    const float2 n = mul2(y.get(2 * i), both(r));
                    dy.set(2 * i, mul2(both(r), fma2(n, both(-c1), mul2(dt, b[i]))));
                    float2 &sum = sum_n[Y ? v : 0][i];
                    sum = fma2(dt, n, sum);
                }
            }
            store_vec<T>(a.dX, row, d, q, dx);
            if (Y) store_vec<T>(a.dY, row, d, q, dy);
        }
    };
    // rows one behind the other, the next on its way; the first one has been asked for. GATE 2: from group to group, each with its end
    auto some_rows = [&](int64_t row, int64_t end, int64_t step) {
        int at = 0;
        int64_t g = first_group, group_end = GATE == 2 ? row + s.group : 0;
#pragma unroll 1
        for (; row < end; row += step) {
            const bool ends = GATE == 2 && (row + 1 == group_end || row + 1 == end);
            ask(row + step, end, at ^ 1, ends ? g + 1 : g);
            copies_wait<1>();
            one_row(row, at);
            if (ends) {
#pragma unroll
                for (int v = 0; v < V; ++v) {  // the group's gate gradient, and its part of dw
                    const int32_t q = lane + 32 * v;
                    if (q >= pieces) break;
                    Vec<T> gv, dg;
                    gv.raw = mine[at * HELD * pieces + TENSORS * pieces + q];
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        float2 &n = sum_n[Y ? v : 0][i], &w = sum_w[GATE == 2 ? v : 0][i];
                        w = fma2(gv.get(2 * i), n, w);
                        dg.set(2 * i, mul2(*reinterpret_cast<const float2 *>(gw + q * N + 2 * i), n));
                        n = both(0.0f);
                    }
                    store_vec<T>(a.dgate, g, d, q, dg);
                }
                ++g;
                group_end += s.group;
            }
            at ^= 1;
        }
        copies_wait<0>();
    };
    auto block_sums = [&](auto &sums, auto done) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t q = lane + 32 * v;
            if (q >= pieces) break;
#pragma unroll
            for (int i = 0; i < P; i += 2) *reinterpret_cast<float4 *>(columns + team * d + q * N + 2 * i) = make_float4(sums[v][i].x, sums[v][i].y, sums[v][i + 1].x, sums[v][i + 1].y);
        }
        __syncthreads();
        for (int32_t q = threadIdx.x; q < pieces; q += blockDim.x) {  // in the order of the warps
            float2 total[P];
#pragma unroll
            for (int i = 0; i < P; ++i) total[i] = both(0.0f);
#pragma unroll 1
            for (int t = 0; t < s.teams; ++t)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 f = *reinterpret_cast<const float2 *>(columns + t * d + q * N + 2 * i);
                    total[i] = make_float2(total[i].x + f.x, total[i].y + f.y);
                }
            done(q, total);
        }
    };
    auto put = [&](float *part, int32_t q, const float2 (&total)[P]) {
#pragma unroll
        for (int i = 0; i < P; i += 2)
            *reinterpret_cast<float4 *>(part + (int64_t)blockIdx.x * d + (int64_t)q * N + 2 * i) = make_float4(total[i].x, total[i].y, total[i + 1].x, total[i + 1].y);
    };

    some_rows(first, last, GATE == 2 ? 1 : s.teams);
    if (GATE == 2) {
        block_sums(sum_w, [&](int32_t q, const float2 (&total)[P]) { put(part_w, q, total); });
    } else {
        if (Y)
            block_sums(sum_n, [&](int32_t q, const float2 (&total)[P]) {
                if (GATE == 0) {
                    put(part_w, q, total);
                    return;
                }
                const Vec<T> gv = load_vec<T>(a.gate, block_group, d, q);
                float2 w[P], of_w[P];
                load_floats(a.w + (int64_t)q * N, w);
                Vec<T> dg;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    of_w[i] = mul2(gv.get(2 * i), total[i]);
                    dg.set(2 * i, mul2(w[i], total[i]));
                }
                put(part_w, q, of_w);
                if (s.chunks > 1) put(part_gate, q, total);
                else store_vec<T>(a.dgate, block_group, d, q, dg);
            });
    }
    if (NEXT) block_sums(sum_next, [&](int32_t q, const float2 (&total)[P]) { put(part_next, q, total); });
}

// The blocks' sums added up, 32 columns a block, RUNS runs of blocks side by side, eight loads of each in flight, in double and in a fixed order. Blocks of the grid: those of dw, of
// dw_next, then of every gate that several blocks share.
constexpr int RUNS = 32, FEW_CHUNKS = 32;  // gates of few chunks: a block has 32 sums of one run
template <typename T>
__global__ void __launch_bounds__(RUNS * 32) norm_sums_kernel(const NormGradArgs a, const Share s, const float *part_w, const float *part_next, const float *part_gate) {
    wait_previous_kernel();
    __shared__ double sh[RUNS][33];
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const int32_t slabs = (a.d + 31) / 32;
    const int64_t own = (a.y ? 1 : 0) + (a.dNext ? 1 : 0), gates_at = own * slabs;
    if (s.chunks <= FEW_CHUNKS && blockIdx.x >= gates_at) {  // a warp has 32 columns of a gate
        const int64_t number = (blockIdx.x - gates_at) * RUNS + run, g = number / slabs;
        const int32_t at = (int32_t)(number % slabs) * 32 + lane;
        if (g >= s.groups || at >= a.d) return;
        double sum = 0.0;
        for (int64_t b = 0; b < s.chunks; b += 8) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = b + i < s.chunks ? part_gate[(g * s.chunks + b + i) * a.d + at] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += f[i];
        }
        static_cast<T *>(a.dgate)[g * a.d + at] = from_f32<T>((float)(a.w[at] * sum));
        return;
    }
    const int64_t job = blockIdx.x / slabs;
    const int32_t col = (blockIdx.x % slabs) * 32 + lane;
    const float *part = nullptr;
    int64_t from = 0, count = s.blocks, gate_row = -1;
    float *to = nullptr;
    if (a.y && job == 0) { part = part_w; to = a.dw; }
    else if (a.dNext && job == (a.y ? 1 : 0)) { part = part_next; to = a.dw_next; }
    else {
        gate_row = job - own;
        part = part_gate;
        from = gate_row * s.chunks;
        count = s.chunks;
    }
    const int64_t each = (count + RUNS - 1) / RUNS, lo = from + run * each, hi = min(lo + each, from + count);
    double sum = 0.0;
    if (col < a.d)
        for (int64_t b = lo; b < hi; b += 8) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = b + i < hi ? part[(b + i) * a.d + col] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += f[i];
        }
    sh[run][lane] = sum;
    __syncthreads();
    // a warp has one of the columns: its runs in pairs (3001 x 320, both launches: 7.8 us; one behind the other 8.0)
    sum = sh[lane][run];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    const int32_t mine = (blockIdx.x % slabs) * 32 + run;
    if (lane > 0 || mine >= a.d) return;
    if (to) to[mine] = (float)sum;
    else static_cast<T *>(a.dgate)[gate_row * a.d + mine] = from_f32<T>((float)(a.w[mine] * sum));
}

template <typename T, int V> int32_t launch_rows(const NormArgs &a, int warps, int teams, cudaStream_t st) {
    // As many blocks as the SMs hold at once, 3 (bf16, norm and residual, two vectors a lane) or 4 an SM, for several rows each: 32768 x 512 with norm and next 23.4 us (4 an SM: 27.9),
    // 131072 x 512, norm_in 43.3 (3: 45.5, 6: 48.6), 65536 x 256 23.7 (26.1, 27.8), float, 30000 x 320 29.4 (31.5, 32.7). Blocks of one row a team: 26.8, 55.0, 31.5 and 38.6; they stay for few
    // rows and for rows of more than eight warps (8192 x 8192, norm, no gate, next: 121, several rows each 131).
    const int64_t at_once = 148 * (V == 2 && a.y && sizeof(T) == 2 ? 3 : 4), blocks = cdiv(a.T, teams);
    const bool ahead = V <= 2 && warps <= 8 && blocks > at_once;
    const dim3 grid((unsigned)(ahead ? at_once : blocks)), block(warps * 32 * teams);
#define MOE_NORM_ROWS(Y, NEXT, GATE)                                                                                      \
    do {                                                                                                                  \
        if constexpr (V <= 2) {                                                                                           \
            if (ahead) {                                                                                                  \
                launch_kernel(norm_rows_kernel<T, V, Y, NEXT, GATE, true>, grid, block, 0, st, a, warps);                 \
                break;                                                                                                    \
            }                                                                                                             \
        }                                                                                                                 \
        launch_kernel(norm_rows_kernel<T, V, Y, NEXT, GATE, false>, grid, block, 0, st, a, warps);                        \
    } while (0)
    if (a.y && a.next && a.gate) MOE_NORM_ROWS(true, true, true);
    else if (a.y && a.next) MOE_NORM_ROWS(true, true, false);
    else if (a.y && a.gate) MOE_NORM_ROWS(true, false, true);
    else if (a.y) MOE_NORM_ROWS(true, false, false);
    else MOE_NORM_ROWS(false, true, false);
#undef MOE_NORM_ROWS
    MOE_LAUNCHED();
    return MOE_OK;
}

template <typename T, int V> int32_t launch_grads(const NormGradArgs &a, const Share &s, cudaStream_t st) {
    const int64_t most = s.most * a.d;
    float *part_w = a.ws, *part_next = part_w + most, *part_gate = part_next + most;
    if (s.blocks > 0) {
        const dim3 grid((unsigned)s.blocks), block(s.warps * 32 * s.teams);
        const bool few = a.gate && s.chunks == 0;
        const int tensors = (a.y ? 2 : 1) + (a.dNext ? 2 : 0);
        size_t shared = 0;
        if (s.ring) shared = sizeof(float) * a.d * ((a.y ? 1 : 0) + (a.dNext ? 1 : 0)) + (size_t)s.teams * RING_ROWS * (tensors + (few ? 1 : 0)) * a.d * sizeof(T);
        auto launch = [&](auto *kernel, PerDevice &allowed) -> int32_t {
            if (s.ring && !allow_shared(allowed, kernel, SHARED_ALLOWED)) return MOE_ERR_CUDA;
            launch_kernel(kernel, grid, block, shared, st, a, s, part_w, part_next, part_gate);
            return MOE_OK;
        };
#define MOE_NORM_GRADS(Y, NEXT, GATE)                                                     \
    do {                                                                                  \
        static PerDevice allowed;                                                         \
        if constexpr (V <= 4) {                                                           \
            if (s.ring) {                                                                 \
                MOE_TRY(launch(norm_stream_kernel<T, V, Y, NEXT, GATE>, allowed));        \
                break;                                                                    \
            }                                                                             \
        }                                                                                 \
        MOE_TRY(launch(norm_grads_kernel<T, V, Y, NEXT, GATE>, allowed));                 \
    } while (0)
        if (a.y && a.dNext && few) MOE_NORM_GRADS(true, true, 2);
        else if (a.y && a.dNext && a.gate) MOE_NORM_GRADS(true, true, 1);
        else if (a.y && a.dNext) MOE_NORM_GRADS(true, true, 0);
        else if (a.y && few) MOE_NORM_GRADS(true, false, 2);
        else if (a.y && a.gate) MOE_NORM_GRADS(true, false, 1);
        else if (a.y) MOE_NORM_GRADS(true, false, 0);
        else MOE_NORM_GRADS(false, true, 0);
#undef MOE_NORM_GRADS
        MOE_LAUNCHED();
    }
    const int64_t slabs = cdiv(a.d, 32), gates = a.gate && s.chunks > 1 ? s.groups * slabs : 0;
    launch_kernel(norm_sums_kernel<T>, dim3((unsigned)(((a.y ? 1 : 0) + (a.dNext ? 1 : 0)) * slabs + (s.chunks <= FEW_CHUNKS ? cdiv(gates, RUNS) : gates))), dim3(RUNS * 32), 0, st, a, s, (const float *)part_w, (const float *)part_next, (const float *)part_gate);
    MOE_LAUNCHED();
    return MOE_OK;
}

}  // namespace

int64_t norm_grad_floats(int64_t T, int32_t d, int32_t act) {
    int64_t most = 0;
    for (int tensors = 2; tensors <= 5; ++tensors) {
        int warps, teams, V, ring;
        grad_team_of(d, act, tensors, &warps, &teams, &V, &ring);
        most = imax(most, most_blocks(T, teams));
    }
    return 3 * most * d;
}

int32_t launch_norms(const NormArgs &a, cudaStream_t st) {
    if (a.T == 0) return MOE_OK;
    int warps, teams, V;
    team_of(a.d, a.act, &warps, &teams, &V);
    if (a.act == MOE_BF16) return V == 1 ? launch_rows<bf16, 1>(a, warps, teams, st) : V == 2 ? launch_rows<bf16, 2>(a, warps, teams, st) : launch_rows<bf16, 4>(a, warps, teams, st);
    return V == 1 ? launch_rows<float, 1>(a, warps, teams, st) : V == 2 ? launch_rows<float, 2>(a, warps, teams, st) : V == 4 ? launch_rows<float, 4>(a, warps, teams, st) : launch_rows<float, 8>(a, warps, teams, st);
}

int32_t launch_norm_grads(const NormGradArgs &a, cudaStream_t st) {
    const Share s = share_of(a.T, a.d, a.act, (a.y ? 2 : 1) + (a.dNext ? 2 : 0), a.gate ? a.rows_per_gate : 0);
    if (a.act == MOE_BF16) return s.V == 1 ? launch_grads<bf16, 1>(a, s, st) : s.V == 2 ? launch_grads<bf16, 2>(a, s, st) : launch_grads<bf16, 4>(a, s, st);
    return s.V == 1 ? launch_grads<float, 1>(a, s, st) : s.V == 2 ? launch_grads<float, 2>(a, s, st) : s.V == 4 ? launch_grads<float, 4>(a, s, st) : launch_grads<float, 8>(a, s, st);
}

}  // namespace moe
