"""Host side of the gated-delta core's workspaces (no GPU): what the entry point refuses needs none."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def m():
    if not os.path.exists(os.path.join(ROOT, "paper_2506_01206_amd", "libmamba_hip.so")):
        from paper_2506_01206_amd import build
        build.build()
    from paper_2506_01206_amd import binding
    return binding


@pytest.mark.parametrize("batch,L,H,Hk,P,N", [
    (70000, 100, 8, 4, 64, 128), (1, 100, 70000, 1, 64, 128), (1025, 100, 512, 4, 64, 128), (1, (1 << 31) + 1, 8, 4, 64, 128), (1 << 43, 512, 1, 1, 64, 64),
    (1 << 30, 64, 1 << 15, 1, 64, 64), (1, 100, 8, 3, 64, 128), (1, 100, 8, 4, 32, 128), (1, 100, 8, 0, 64, 128), (-1, 100, 8, 4, 64, 128)])
def test_no_workspace_for_what_is_refused(m, batch, L, H, Hk, P, N):
    """0 is the documented answer for an unsupported shape; beyond the limits the size itself overflows."""
    at = [(i + 1) << 50 for i in range(13)]
    status = m.lib.mamba_gated_delta_fwd(*at, 1 << 49, batch, L, H, Hk, P, N, 1.0, 1e-6, 1, 1, 1, 1, None)
    assert status in (m.STATUS["UNSUPPORTED"], m.STATUS["BAD_SHAPE"])
    assert m.mamba_gated_delta_workspace_bytes(batch, L, H, Hk, P, N) == 0


# The plan of a chunked context (csrc/routes.h) against what its launches read and write, written down again here from the kernels' indexing: every
# region of the workspace ends where the next begins, and every grid stays below 2^32 threads a dimension.
SHIM = """
#include "routes.h"
#include <stdio.h>
using namespace mamba;
extern "C" int sweep_one(int64_t B, int64_t L, int64_t H, int64_t Hk, int64_t P, int64_t N, int64_t *seen)
{
    const DeltaPlan p = delta_plan(B, L, H, Hk, P, N);
    const int64_t heads = B * H, state = heads * P * N * 4;
    auto fail = [&](const char *what, int64_t a, int64_t b) {
        printf("%s: %lld %lld, B=%lld L=%lld H=%lld Hk=%lld P=%lld N=%lld\\n", what, (long long)a, (long long)b, (long long)B, (long long)L, (long long)H, (long long)Hk,
               (long long)P, (long long)N);
        return 1;
    };
    if (p.slab < 1 || p.part < 1 || p.chunks * 64 < L || (p.chunks - 1) * 64 >= L) return fail("chunks", p.chunks, p.slab);
    const int64_t at[] = {0, p.frags_at, p.raw_at, p.state_at, p.parts_at, p.map_at, p.bytes};
    for (int i = 0; i < 6; ++i)
        if (at[i] > at[i + 1] || at[i] % 16) return fail("regions", i, at[i]);
    int64_t chunks = 0, slabs = 0;
    for (int64_t first = 0; first < p.chunks; first += p.slab, ++slabs) {
        const DeltaSlab s = delta_slab(p, first);
        const int64_t n = s.chunks, last = first + n == p.chunks;
        chunks += n;
        // the preparation: a block of the workspace to a chunk and head, 37888 bytes; fragments of K and Q to a chunk and key head
        if (((heads - 1) * n + n) * 37888 > p.frags_at) return fail("X", n, p.frags_at);
        if (((B * Hk - 1) * n + n) * 2 * N * 64 * 2 > p.raw_at - p.frags_at) return fail("fragments", n, p.raw_at);
        if (((B - 1) * n + n) * 64 * H * P * 4 > p.state_at - p.raw_at) return fail("outputs ahead of the norm", n, p.state_at);
        if (!last && state > p.parts_at - p.state_at) return fail("state between slabs", state, p.parts_at);
        // parts: all of them have chunks; starts of those from the second on; maps of all but the first and the last
        if (s.parts < 1 || (s.parts - 1) * p.part >= n || s.parts * p.part < n) return fail("parts", s.parts, p.part);
        if ((s.parts - 1) * state > p.map_at - p.parts_at) return fail("starts", s.parts, p.map_at);
        if (s.maps != (s.parts > 2 ? s.parts - 2 : 0) || s.maps * heads * N * N * 4 > p.bytes - p.map_at) return fail("maps", s.maps, p.bytes);
        // grids (threads of a dimension), a walk's numbers in 32 bits, tokens of a part as int
        const int64_t first_walk = delta_walk_blocks(heads, P, N, 1, s.maps), then = delta_walk_blocks(heads, P, N, s.parts - 1, 0);
        if (first_walk * 512 >= (int64_t)1 << 32 || then * 512 >= (int64_t)1 << 32) return fail("walk", first_walk, then);
        if (heads * (s.parts > 1 ? s.parts - 1 : 1) * 8 * (P + N) / 16 >= (int64_t)1 << 32) return fail("numbers", s.parts, 0);
        if (n * 512 >= (int64_t)1 << 32 || H > 65535 || B > 65535) return fail("preparation", n, H);
        if (heads * P / 16 * 4 * N >= (int64_t)1 << 32) return fail("join", heads, P);
        const int64_t quads = (last ? L - first * 64 : n * 64) * H * P / 4;
        if ((quads + 255) / 256 * 256 >= (int64_t)1 << 32) return fail("norm", quads, 0);
        if (p.part * 64 >= (int64_t)1 << 31 || 64 * H * P >= (int64_t)1 << 32 || 64 * Hk * N >= (int64_t)1 << 32) return fail("offsets", p.part, H);
        ++seen[s.parts > 3 ? 3 : s.parts - 1];
    }
    if (chunks != p.chunks) return fail("slabs", chunks, p.chunks);
    ++seen[slabs > 1 ? 5 : 4];
    return 0;
}
// every workgroup of a walk has one place and every place one, as the kernel takes its number apart; and the fullest XCD has as many as is said
extern "C" int walk_places(int64_t heads, int64_t P, int64_t N, int64_t walked, int64_t maps)
{
    const uint32_t values = P / 16, walks = (heads * walked + 7) / 8 * 8 * values;
    const int64_t blocks = delta_walk_blocks(heads, P, N, walked, maps), places = heads * walked * values + heads * maps * (values + N / 16);
    static char seen[1 << 22];
    if (places > (1 << 22)) return 2;
    for (int64_t i = 0; i < places; ++i) seen[i] = 0;
    int64_t found = 0, xcd[8] = {0};
    for (uint32_t id = 0; id < blocks; ++id) {
        const bool map = id >= walks;
        const uint32_t index = map ? id - walks : id, each = map ? values + N / 16 : values, place = index >> 3;
        const uint32_t pair = place / each * 8 + ((map ? index - (uint32_t)(heads * walked) : index) & 7), block = place % each, turn = pair / heads;
        if (turn >= (map ? maps : walked)) continue;
        const int64_t at = map ? heads * walked * values + ((int64_t)pair * each + block) : (int64_t)pair * each + block;
        if (at >= places || seen[at]) return 1;
        seen[at] = 1, ++found, ++xcd[id & 7];
    }
    int64_t most = 0;
    for (int i = 0; i < 8; ++i) most = xcd[i] > most ? xcd[i] : most;
    return found != places || most != delta_fullest_xcd(heads, P, N, walked, maps);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    import ctypes
    import subprocess
    d = tmp_path_factory.mktemp("plan")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-shared", "-fPIC",
                           "-o", str(d / "shim.so"), "-I" + os.path.join(ROOT, "paper_2506_01206_amd", "csrc"), str(d / "shim.cpp")])
    lib = ctypes.CDLL(str(d / "shim.so"))
    lib.sweep_one.argtypes = [ctypes.c_int64] * 6 + [ctypes.c_void_p]
    lib.walk_places.argtypes = [ctypes.c_int64] * 5
    return lib


def test_the_launches_of_a_plan_stay_in_its_regions(plan):
    import ctypes
    import random
    rng = random.Random(1)
    seen = (ctypes.c_int64 * 6)()
    lengths = [1, 7, 64, 65, 100, 1000, 2048, 8191, 32768, 131142, 1 << 20, (1 << 31) - 1, 1 << 31]
    cases = [(B, L, H, Hk) for B in (1, 2, 8, 65535) for L in lengths for H, Hk in ((1, 1), (2, 1), (8, 8), (24, 24), (32, 8), (128, 1), (65535, 1))]
    cases += [(B, int(2 ** rng.uniform(0, 20)), H * g, H) for _ in range(3000) for B, H, g in
              ((int(2 ** rng.uniform(0, 6)), int(2 ** rng.uniform(0, 6)), rng.choice((1, 2, 3, 4, 8))),)]
    cases += [(1, L, 4, 2) for L in range(1, 70000, 61)]         # last slabs and parts of all lengths
    for B, L, H, Hk in cases:
        if B * H <= 1 << 19 and B * L * H < 1 << 45:
            for N, P in ((64, 64), (64, 128), (128, 64), (128, 128)):
                if L < 1 << 24 or B * H >= 64:                   # (fewer heads have no more slabs to show, only more of them to go through)
                    assert plan.sweep_one(B, L, H, Hk, P, N, seen) == 0
    assert min(seen) > 0, list(seen)                             # slabs of one, two, three and more parts; one slab and several


def test_every_workgroup_of_a_walk_has_a_place(plan):
    for heads in list(range(1, 41)) + [63, 64, 65, 128, 255, 512]:
        for N, P in ((64, 64), (64, 128), (128, 64), (128, 128)):
            for walked, maps in [(1, 0), (1, 1), (2, 0), (1, 3), (4, 0), (1, 7), (1, 8), (9, 0), (1, 14)]:
                assert plan.walk_places(heads, P, N, walked, maps) == 0, (heads, N, P, walked, maps)
