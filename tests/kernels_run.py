"""The library's kernels that a call launched, as the driver's tracing interface reports them."""
import json
import os
import re
import tempfile

import pytest
import torch
from torch.profiler import ProfilerActivity, profile


def kernels_of(call):
    """[(name, [template arguments], blocks)] of the library's launches in call()."""
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    with tempfile.TemporaryDirectory() as d:
        p.export_chrome_trace(os.path.join(d, "trace.json"))
        with open(os.path.join(d, "trace.json")) as f:
            events = [e for e in json.load(f)["traceEvents"] if e.get("cat") == "kernel"]
    if not events:
        pytest.skip("launches cannot be traced here")
    found = []
    for e in events:
        m = re.match(r"(?:void )?adloco::(?:\(anonymous namespace\)::)?(\w+)(?:<([^(]*?)>)?\(", e["name"])
        if m:
            x, y, z = e["args"]["grid"]
            found.append((m.group(1), [a.strip() for a in (m.group(2) or "").split(",")], x * y * z))
    return found
