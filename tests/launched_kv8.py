"""Names of the kernels that an attention over the 8-bit cache launches.

A process of its own, as in launched_kernels.py: a process that has profiled once can lose kernels in a later profile."""
import json
import subprocess
import sys
import time


def launched_kv8(cases):
    """cases: list of (heads, KV heads, head dimension, requests, rows, context, block, format) -> list of texts, the kernels' names."""
    r = subprocess.run([sys.executable, __file__], input=json.dumps(cases), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return json.loads(r.stdout.splitlines()[-1])


if __name__ == "__main__":
    import os
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    import torch
    from paper_2608_26140_b200 import binding as ab

    calls = []
    for H, hkv, d, B, n, T, block, fmt in json.load(sys.stdin):
        ctx = ab.Context(max(hkv * d, 128), H, hkv, d, 128, 1e-5, 0, B, T, 0, 1, 0, "cuda:0")
        keep, cache = ctx.new_kv8(B, T, block, fmt)
        q = torch.zeros((B, n, H, d), dtype=torch.bfloat16, device="cuda:0")
        calls.append((ctx, keep, cache, B, T, q, torch.empty_like(q)))
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        time.sleep(0.05)                             # room on both sides of the kernels for the two clocks to differ
        for ctx, keep, cache, B, T, q, o in calls:
            ctx.kv8_attention(cache, B, T, q, o)
            torch.cuda.synchronize()
        time.sleep(0.05)
    kernels = sorted((e.time_range.start, e.name) for e in prof.events() if "kv8" in e.name)
    assert len(kernels) == len(calls), kernels
    print(json.dumps([name for _, name in kernels]))
