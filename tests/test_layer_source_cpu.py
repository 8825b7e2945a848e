"""What the sources of the decoder-layer kernels have to keep, where a run on the GPU could not show a violation safely."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2407_04480_b200", "csrc")


def kernels():
    """(name, body) of every __global__ function of the layer library."""
    for unit in sorted(f for f in os.listdir(CSRC) if f.startswith("layer_") and f.endswith(".cu")):
        text = open(os.path.join(CSRC, unit)).read()
        for m in re.finditer(r"__global__ void (?:__launch_bounds__\([^{;]*?\)\s+)?(\w+)\(", text):
            at = text.index("{\n", m.end())
            yield m.group(1), text[at:text.index("\n}\n", at)]


def test_every_kernel_waits_for_the_launch_before_it_touches_memory():
    """Launched so that it may start under the launch before, a kernel is promised that launch's results, and those of the
    ones before it, only behind its own wait: every thread has to pass one, unconditionally, ahead of the first access."""
    touches = re.compile(r"query_rows\(P|key_rows\(P|load_box\(|load_tile<|fetch\(t\)|P\.(?:lse|row_dot|in_counts|dlosses|positions|table|mask)\b|table\[")
    seen = 0
    for name, body in kernels():
        wait = re.search(r"^    wait_for_previous\(\);$", body, re.M)
        assert wait, name + " has no unconditional wait"
        asked = re.search(r"no_such_rows\(P", body)          # waits itself
        first = touches.search(re.sub(r"const auto fetch = .*", lambda m: " " * len(m.group()), body))
        assert first is None or first.start() > min(wait.start(), asked.start() if asked else len(body)), name
        seen += 1
    assert seen >= 7
