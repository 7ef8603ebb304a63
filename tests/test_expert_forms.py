"""Host-only: every kernel of the 8-bit expert layer and of the expert layer's gradients is chosen for a case of the GPU tests.  The launch
rules' own source is compiled against stand-ins for the launches, so that a threshold that moves cannot leave a kernel without a
test."""
import ctypes
import os
import subprocess

import pytest

import paper_2411_00662_amd as m
from paper_2411_00662_amd.build import CSRC

STAND_INS = r"""
#include <algorithm>
#include <cstdint>
#include <set>
#include <string>
#include <type_traits>
namespace {
enum { MONTA_OK = 0, MONTA_ERR_UNSUPPORTED = -2 };
struct ExpertArgs { int16_t E; int8_t spread; int32_t H, N; };
struct GradArgs { ExpertArgs a; const void *dx, *dw; };
struct Expert8Args { ExpertArgs a; int32_t nb; };
typedef void *hipStream_t;
constexpr int kBig8 = 256;
std::set<std::string> &known() { static std::set<std::string> s; return s; }
std::string chosen;
template <typename F> std::string name_of()
{
    const std::string s = __PRETTY_FUNCTION__;
    const size_t at = s.find("F = ") + 4;
    return s.substr(at, s.find_first_of(";]", at) - at);
}
template <typename F> struct Kernel { static bool is_known; };
template <typename F> bool Kernel<F>::is_known = known().insert(name_of<F>()).second;
template <typename F> int chose() { (void)Kernel<F>::is_known; chosen += name_of<F>() + "\n"; return MONTA_OK; }
bool launchable(int64_t, int) { return true; }

template <typename Derived> struct Tiles { static int64_t grid(const ExpertArgs &, int64_t) { return 1; } };
template <bool DW, int RB, int CB, bool LAST = false> struct Wide : Tiles<Wide<DW, RB, CB, LAST>> {};
template <int XR, int CW, int NST> struct Short : Tiles<Short<XR, CW, NST>> {};
template <int NST> struct Slim : Tiles<Slim<NST>> {};
template <bool DW, int BR, int NST> struct F32 : Tiles<F32<DW, BR, NST>> {};
template <typename A, typename B> struct Both {};
template <typename Form> int launch_form(const GradArgs &, int64_t, hipStream_t) { return chose<Form>(); }
template <typename Dx, typename Dw> int launch_both(const GradArgs &, int64_t, hipStream_t) { return chose<Both<Dx, Dw>>(); }

template <int XR, int WR, int WX, int WW, int NST, bool F32> struct Ring8 {};
template <int CB, int W, int D, bool F32> struct Split8 {};
template <bool LAST, bool TAIL> struct Big8 {};
template <int XR, int WR, int WX, int WW, int NST, bool F32> int launch_expert8(const void *, const void *, void *, const Expert8Args &, int64_t, hipStream_t)
{ return chose<Ring8<XR, WR, WX, WW, NST, F32>>(); }
template <int CB, int W, int D, bool F32> int launch_expert8_split(const void *, const void *, void *, const Expert8Args &, int64_t, hipStream_t)
{ return chose<Split8<CB, W, D, F32>>(); }
template <bool LAST, bool TAIL> int launch_expert8_big_k(const void *, const void *, void *, const Expert8Args &, int64_t, hipStream_t)
{ return chose<Big8<LAST, TAIL>>(); }
"""
CALLS = r"""
}
extern "C" {
const char *known_kernels()
{
    static std::string s;
    s.clear();
    for (const auto &k : known()) s += k + "\n";
    return s.c_str();
}
const char *grad_kernels(int E, int H, int N, int bf16, long long rows, int dx, int dw)
{
    chosen.clear();
    launch_grads(GradArgs{{(int16_t)E, 0, H, N}, dx ? &chosen : nullptr, dw ? &chosen : nullptr}, bf16, rows, nullptr);
    return chosen.c_str();
}
const char *expert8_kernels(int E, int H, int N, int bf16, long long rows, long long kept, int slice)
{
    chosen.clear();
    const Expert8Args b{{(int16_t)E, 0, H, N}, (H + 127) / 128};
    if (bf16) launch_expert8_tiled<false>(nullptr, nullptr, nullptr, b, rows, kept, slice, nullptr);
    else launch_expert8_tiled<true>(nullptr, nullptr, nullptr, b, rows, kept, slice, nullptr);
    return chosen.c_str();
}
}
"""


def function(source, signature):
    text = open(os.path.join(CSRC, source)).read()
    at = text.index(signature)
    return text[at:text.index("\n}\n", at) + 3]


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    src, lib = str(d / "rules.cpp"), str(d / "librules.so")
    with open(src, "w") as f:
        f.write(STAND_INS + function("monta_grad.hip", "int launch_grads(")
                + "template <bool RAGGED_LAST>\n" + function("monta_expert8.hip", "int launch_expert8_big(")
                + "template <bool F32>\n" + function("monta_expert8.hip", "int launch_expert8_tiled(") + CALLS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-shared", "-fPIC", "-o", lib, src], check=True)
    so = ctypes.CDLL(lib)
    for name in ("known_kernels", "grad_kernels", "expert8_kernels"):
        getattr(so, name).restype = ctypes.c_char_p
    so.grad_kernels.argtypes = [ctypes.c_int] * 4 + [ctypes.c_longlong] + [ctypes.c_int] * 2
    so.expert8_kernels.argtypes = [ctypes.c_int] * 4 + [ctypes.c_longlong] * 2 + [ctypes.c_int]
    return so


def kept_bound(T, E, k, cf):
    L = m.monta_ws_layout_query(m.make_cfg(T, 16, m.BF16, E, k, 1, 1, 1, cf))
    return min(T * k, E * L.capacity)


def names(text):
    return {n for n in text.decode().split("\n") if n}


def test_gradients(rules):
    """All kernels of the gradients: joined launches and, where one gradient is asked for or both go out apart, single ones."""
    import test_gpu_expert_forms as forms
    import test_gpu_expert_grad as grads
    reached = set()
    for T, H, N, E, k, cf, *_ in grads.CASES + grads.LONG + forms.GRADS:
        for bf16 in (0, 1):
            reached |= names(rules.grad_kernels(E, H, N, bf16, kept_bound(T, E, k, cf), 1, 1))
    alone = [(len(loads), H, N, sum(loads)) for loads, H, N in forms.GRADS_TO]
    alone += [(E, H, N, kept_bound(T, E, k, cf)) for T, H, N, E, k, cf, *_ in forms.GRADS + grads.CASES[-4:-3] + [(150, 136, 200, 4, 2, 0.8)]]
    for E, H, N, rows in alone:
        for bf16 in (0, 1):
            for dx, dw in ((1, 1), (1, 0), (0, 1)):
                reached |= names(rules.grad_kernels(E, H, N, bf16, rows, dx, dw))
    known = {n for n in names(rules.known_kernels()) if "8<" not in n}
    assert len(known) >= 18 and reached <= known
    assert known - reached == set()


def test_experts8(rules):
    import test_gpu_expert8 as experts8
    import test_gpu_expert_forms as forms
    reached = set()
    for T, H, N, E, k, cf, padded, S, *_ in experts8.CASES + forms.EXPERTS8:
        kept = kept_bound(T, E, k, cf)
        for bf16 in (0, 1):
            reached |= names(rules.expert8_kernels(E, H, N, bf16, kept, kept, -1))
    for loads, H, N in forms.EXPERTS8_TO:
        for bf16 in (0, 1):
            reached |= names(rules.expert8_kernels(len(loads), H, N, bf16, sum(loads), sum(loads), -1))
    known = {n for n in names(rules.known_kernels()) if "8<" in n}
    assert len(known) >= 14 and reached <= known
    assert known - reached == set()


def test_segments_of_every_length(rules):
    """The cases with chosen segments do take the large tiles that they are for: in place and last."""
    import test_gpu_expert_forms as forms
    for loads, H, N in forms.GRADS_TO:
        got = names(rules.grad_kernels(len(loads), H, N, 1, sum(loads), 1, 0))
        assert any(n.endswith("Wide<false, 8, 8, true>" if loads is forms.LAST else "Wide<false, 8, 8>") for n in got), got
    for loads, H, N in forms.EXPERTS8_TO:
        got = names(rules.expert8_kernels(len(loads), H, N, 1, sum(loads), sum(loads), -1))
        want = "Big8<%s, %s>" % (str(loads is forms.LAST).lower(), str(H % 128 != 0).lower())
        assert any(n.endswith(want) for n in got), got
