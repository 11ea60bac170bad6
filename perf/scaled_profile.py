"""What profiles/scaled_kernels.md is made with.

    python perf/scaled_profile.py cases N    N passes of every listed case of
                                             operators.py, inputs resident
    python perf/scaled_profile.py layer      the layer in 8 bits beside the bf16
                                             forward, a line per shape and batch
    python perf/scaled_profile.py table DIR  the table of kernels, from rocprofv3's
                                             outputs for `cases` under DIR: a
                                             kernel trace of 10 passes (DIR/trace)
                                             and counters of 4 (DIR/sq, DIR/fetch,
                                             DIR/write)
"""
import collections
import csv
import glob
import os
import re
import statistics
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2410_12247_amd import moe, synth  # noqa: E402
from perf import operators  # noqa: E402

KERNELS = re.compile(r"((?:tile|stream|mid|norm_quant)_kernel<[^>]*>)")


def cases(passes):
    operators.own = True
    for case in operators.listed():
        state = operators.prepare(case, 1)
        for _ in range(passes):
            operators.run(state)
        torch.cuda.synchronize()
        print(case["name"], flush=True)


def captured(call):
    """us per call, ten of them in a graph (which caller's Python does not slow)."""
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(10):
            call()
    times = []
    for _ in range(9):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        graph.replay()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 100)
    return statistics.median(times)


def quantised(w):
    q = torch.empty(w.shape, dtype=torch.uint8, device="cuda")
    s = torch.empty(w.shape[:-2] + (-(-w.shape[-2] // 128), moe.scale_pitch(w.shape[-1])),
                    dtype=torch.uint8, device="cuda")
    moe.quant_weights(w, q, s)
    return q, s


def layer():
    for name, shape in (("Mixtral shard", "mixtral"), ("DBRX shard", "dbrx"),
                        ("DeepSeekV2 share", "zipf"),
                        ("DeepSeekV2 share, shared experts", "dsv2")):
        c = synth.SHAPES[shape]
        H, I, Is, E, EL, k = c.H, c.I, c.shared_inter, c.E, c.EL, c.k
        shapes = [(EL, I, H), (EL, I, H), (EL, H, I)]
        shapes += [(Is, H), (Is, H), (H, Is)] if Is else []
        weights = [(torch.randn(n, device="cuda") * 0.02).bfloat16() for n in shapes]
        pairs = [quantised(w) for w in weights]
        router = torch.randn(E, H, device="cuda") * 0.02
        for T in (1, 64, 1024, 4096, 16384):
            d = moe.dims(T, H, I, E, k, 0, EL, shared_inter=Is)
            packed = moe.scaled_weights(d, *pairs)
            x = torch.randn(T, H, device="cuda").bfloat16()
            y = torch.empty(T, H, device="cuda")
            ws = torch.empty(moe.forward_scaled_bytes(d), dtype=torch.uint8, device="cuda")
            bf16 = moe.MoEBuffers(d, moe.opts())
            scaled = captured(lambda: moe.forward_scaled(d, x, None, None, 1e-6, None, router, None,
                                                         packed, y, None, None, None, ws))
            plain = captured(lambda: bf16.run(x, router, None, *weights))
            off = float((y - bf16.y).norm() / bf16.y.norm())
            print(f"{name}, tokens {T}: {scaled:.0f} / {plain:.0f} us, off by {100 * off:.1f}%",
                  flush=True)


def rows_of(pattern):
    with open(glob.glob(pattern, recursive=True)[0]) as f:
        return list(csv.DictReader(f))


def microseconds(r):
    return (int(r["End_Timestamp"]) - int(r["Start_Timestamp"])) / 1e3


def by_case(launches, passes):
    """(case, kernel's name, its launches) of the launches in order."""
    out, i = [], 0
    for case in operators.listed():
        n = 2 if case["op"] == "ffn" else 1
        of = launches[i:i + n * passes]
        i += n * passes
        out += [(case["name"], of[j][0], [v for _, v in of[j::n]]) for j in range(n)]
    assert i == len(launches), (i, len(launches))
    return out


def counted(path):
    launches = collections.OrderedDict()
    for r in rows_of(path + "/**/*counter_collection.csv"):
        m = KERNELS.search(r["Kernel_Name"])
        if m:
            _, v = launches.setdefault(int(r["Dispatch_Id"]), (m.group(1), {"us": microseconds(r)}))
            v[r["Counter_Name"]] = float(r["Counter_Value"])
    return by_case([launches[i] for i in sorted(launches)], 4)


def table(path):
    trace = sorted(rows_of(path + "/trace/**/*kernel_trace.csv"),
                   key=lambda r: int(r["Start_Timestamp"]))
    traced = [(KERNELS.search(r["Kernel_Name"]), r) for r in trace]
    times = by_case([(m.group(1), microseconds(r)) for m, r in traced if m], 10)
    sq, fetch, write = (counted(f"{path}/{n}") for n in ("sq", "fetch", "write"))
    print("| case | kernel | us | read MB | written MB | TB/s | MFMA busy | GHz | LDS conflicts |")
    print("|---|---|---|---|---|---|---|---|---|")
    for i, (case, kernel, us) in enumerate(times):
        def of(run, counter):
            return statistics.median(v[counter] for v in run[i][2][1:])
        t = statistics.median(us[1:])
        read, written = of(fetch, "FETCH_SIZE") * 2048 / 1e6, of(write, "WRITE_SIZE") * 1024 / 1e6
        line = f"| {case} | `{kernel}` | {t:.1f} | {read:.1f} | {written:.1f} | " \
               f"{(read + written) / t:.2f} | "
        if t > 50:
            cycles = of(sq, "GRBM_GUI_ACTIVE") / 8
            line += f"{of(sq, 'SQ_VALU_MFMA_BUSY_CYCLES') / 1024 / cycles:.0%} | " \
                    f"{cycles / of(sq, 'us') / 1e3:.2f} | " \
                    f"{of(sq, 'SQ_LDS_BANK_CONFLICT') / of(sq, 'SQ_BUSY_CU_CYCLES') * 1e3:.0f} |"
        else:
            line += "- | - | - |"
        print(line)


if __name__ == "__main__":
    if sys.argv[1] == "cases":
        cases(int(sys.argv[2]))
    elif sys.argv[1] == "layer":
        layer()
    else:
        table(sys.argv[2])
