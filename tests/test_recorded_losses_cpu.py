"""What the row operators and the training step's losses launch, without a GPU:
tests/recorded_losses.cpp drives them over many sizes and writes their buffers down."""
import os
import subprocess

import pytest

from paper_2608_19889_amd import axon, build
from test_recorded_cpu import HERE, Launch, Limit, _event


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    axon.lib()
    exe = str(tmp_path_factory.mktemp("recorded") / "recorded_losses")
    pkg = os.path.dirname(axon.LIB_PATH)
    subprocess.run([build.HIPCC, *[f for f in build.FLAGS if f not in ("-O3", "-fPIC")], "--offload-host-only", "-x",
                    "hip", os.path.join(HERE, "recorded_losses.cpp"), "-rdynamic", "-o", exe, "-L" + pkg,
                    "-l:" + os.path.basename(axon.LIB_PATH), "-Wl,-rpath," + pkg],
                   check=True, capture_output=True, text=True)

    def run(scenario):
        r = subprocess.run([exe, scenario], capture_output=True, text=True, timeout=100)
        assert r.returncode == 0 and r.stdout.endswith("done\n"), r.stdout[-500:] + r.stderr[-500:]
        return [_event(line) for line in r.stdout.splitlines()[:-1]]
    return run


@pytest.mark.parametrize("scenario,least", [("operators", 5000), ("steps", 300)])
def test_what_the_kernels_keep_stays_inside_its_buffer(recorder, scenario, least):
    """Partial rows, statistics, coefficients and sequences' sums lie inside one
    allocation of the model, or inside a workspace of exactly the bytes that its
    operator asks for."""
    ends, step, seen = {}, "", 0
    bases = []
    for e in recorder(scenario):
        if isinstance(e, (Launch, Limit)):
            continue
        if e[0] == "alloc":
            ends[e[1]] = e[1] + e[2]
            bases.append(e[1])  # (addresses only grow)
        elif e[0] == "mark":
            step = e[1]
        elif e[0] == "parts":
            base = next((b for b in reversed(bases) if b <= e[1]), None)
            assert base is not None and e[1] + e[2] <= ends[base], (step, e, base and ends[base] - e[1])
            seen += 1
    assert seen > least


def test_no_operator_clears_with_a_memset_or_allocates(recorder):
    """Kernels only, so a caller may capture them; of a model's steps that holds from
    the second on (the first lays the training buffers out)."""
    ev = recorder("operators")
    assert sum(isinstance(e, Launch) for e in ev) > 3000
    assert not any(e[0] == "fill" for e in ev if not isinstance(e, (Launch, Limit)))
    step, seen = "", set()
    for e in recorder("steps"):
        if isinstance(e, Launch):
            if step == "second":
                seen |= {k for k in ("preference_finish", "policy_finish", "ln_bwd", "ce_grad") if k in e.kernel}
        elif isinstance(e, Limit):
            assert step != "second"
        elif e[0] == "mark":
            step = e[1]
        else:
            assert step != "second" or e[0] == "parts", e
    assert len(seen) == 4
