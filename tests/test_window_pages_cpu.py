"""Which pages a window leaves out: the kernel's arithmetic, evaluated where signed overflow is an error, against the definition."""
import os
import re
import subprocess

from paper_2401_09670_amd import build

MOST = 2 ** 31 - 1
PAGE = 16


def _program(calls):
    """seen_of as the kernel's source has it, as a constant expression, and a check of each call."""
    with open(os.path.join(build.CSRC, "attn_paged.hip")) as f:
        source = f.read()
    body = re.search(r"struct Seen \{.*?\n\};\n__device__ __forceinline__ Seen seen_of\(.*?\n\}\n", source, re.S).group(0)
    checks = "\n".join(f"static_assert(same(seen_of({length}, {window}, {sinks}), {want}));" for length, window, sinks, want in calls)
    return f"""#define __device__ constexpr
#define __forceinline__
constexpr int kKvPage = {PAGE};
constexpr int max(int a, int b) {{ return a > b ? a : b; }}
constexpr int min(int a, int b) {{ return a < b ? a : b; }}
{body}
constexpr bool same(Seen s, int sink_pages, int sink_len, int gap, int low) {{
  return s.sink_pages == sink_pages && s.sink_len == sink_len && s.gap == gap && s.low == low;
}}
{checks}
int main() {{}}
"""


def _want(length, window, sinks):
    hidden = max(length - window, 0)
    if sinks >= hidden:
        return "0, 0, 0, 0"
    pages = -(-sinks // PAGE)
    return f"{pages}, {sinks}, {hidden // PAGE - pages}, {hidden % PAGE}"


def test_no_length_or_window_overflows():
    """Lengths below 0 stand for lanes that have no sequence."""
    lens = [-2 * PAGE, -1, 0, 1, 15, 16, 17, 100, 5000, MOST - 1024]
    windows = [1, 2, 16, 33, 4096, MOST - 1, MOST]
    calls = [(l, w, s, _want(l, w, s)) for l in lens for w in windows for s in (0, 1, 16, 40, MOST)]
    assert len({c[3] for c in calls}) > 20
    out = subprocess.run([build.CXX, "-std=c++17", "-fsyntax-only", "-x", "c++", "-"], input=_program(calls), capture_output=True,
                         text=True)
    assert out.returncode == 0, out.stderr[:3000]
