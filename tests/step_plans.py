"""Which kernels a call of the loss or of orthogonalising takes: the library's own rules (csrc/loss_plan.h, csrc/orth_plan.h), compiled for the host."""
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TYPES = {"f32": 0, "bf16": 1, "f16": 2}

# (count, rows, cols, type of the result): together every kernel that matrices of 8 to 9000 rows and columns take
ORTH_SHAPES = [
    (1, 17, 17, "bf16"), (1, 17, 17, "f16"), (1, 18, 17, "f16"), (1, 20, 17, "bf16"), (1, 66, 17, "f32"), (1, 67, 17, "bf16"), (1, 18, 65, "f16"),
    (1, 17, 73, "bf16"), (1, 17, 261, "f32"), (1, 262, 17, "f16"), (1, 274, 17, "bf16"), (1, 18, 269, "bf16"), (1, 68, 65, "f16"),
    (1, 66, 68, "bf16"), (1, 1042, 17, "f16"), (1, 17, 1101, "bf16"), (1, 1131, 17, "bf16"), (1, 18, 1041, "f16"), (1, 131, 65, "f16"),
    (1, 65, 134, "bf16"), (1, 66, 131, "f32"), (1, 142, 66, "bf16"), (1, 69, 1193, "f32"), (1, 1487, 65, "f32"), (1, 66, 1903, "bf16"),
    (1, 1848, 73, "bf16"), (5, 1279, 1199, "f32"), (5, 1416, 1538, "f32"), (5, 1506, 1458, "bf16"), (5, 1439, 1553, "bf16"), (2, 3155, 1700, "f32"),
    (5, 1841, 1743, "f32"), (5, 1987, 1748, "bf16"), (5, 1842, 1899, "f32"), (5, 1875, 2075, "bf16"), (1, 8597, 2471, "bf16"), (1, 4280, 4527, "f32"),
    (5, 2532, 5002, "bf16")
]
# (rows, classes, cols, type, with gradients, with padding, aligned): the same of 1 to 200000 rows, 150000 classes and 9000 columns
LOSS_CALLS = [
    (8, 32, 64, "f16", 0, 1, 0), (1, 360, 64, "f32", 1, 1, 1), (4, 104, 64, "f32", 1, 1, 0), (20, 32, 64, "f32", 0, 1, 1),
    (8, 45, 115, "f32", 0, 1, 1), (1, 45, 1600, "f16", 0, 0, 1), (1, 58, 1280, "bf16", 0, 0, 1), (6, 233, 64, "bf16", 0, 0, 1),
    (1, 83, 1401, "f16", 1, 1, 0), (4, 466, 64, "f16", 0, 0, 1), (36, 193, 22, "f32", 0, 0, 0), (1, 262, 616, "bf16", 0, 1, 1),
    (16, 248, 64, "f32", 1, 0, 1), (27, 5003, 301, "f32", 1, 1, 0),
    (35, 28277, 78, "f32", 1, 1, 0), (5, 844, 64, "f32", 1, 1, 0), (120, 100, 23, "f32", 0, 1, 0), (6, 50, 982, "bf16", 1, 1, 0),
    (75, 30, 951, "f32", 0, 1, 1), (1464, 64, 131, "f16", 1, 1, 0), (70, 956, 192, "bf16", 1, 1, 1), (18, 8923, 477, "f32", 1, 0, 0),
    (4303, 38, 832, "f32", 1, 1, 1), (1495, 6451, 20, "f32", 0, 0, 0), (24658, 33, 318, "f32", 1, 1, 1), (32454, 83, 112, "bf16", 1, 0, 0),
    (13032, 1072, 25, "f16", 0, 1, 1), (131, 26886, 105, "f16", 1, 0, 1), (69, 30237, 192, "f32", 0, 1, 1), (837, 6732, 72, "f16", 1, 0, 0),
    (9945, 562, 78, "f32", 1, 0, 1), (718, 9181, 76, "bf16", 1, 1, 0), (225, 29888, 78, "bf16", 1, 1, 1), (41, 4621, 3328, "bf16", 1, 1, 1),
    (59212, 227, 47, "bf16", 0, 1, 0), (32101, 169, 128, "f16", 1, 0, 0), (80, 1766, 5824, "f32", 1, 1, 1), (347, 4639, 512, "bf16", 1, 0, 0),
    (258, 3005, 1152, "f16", 1, 0, 0), (211, 32464, 141, "f16", 1, 1, 0), (93, 60298, 184, "bf16", 1, 0, 0), (2191, 147, 3477, "bf16", 1, 0, 1),
    (83, 58688, 268, "bf16", 0, 1, 1), (21245, 339, 183, "f16", 0, 0, 1), (1361, 7410, 137, "f32", 1, 0, 1), (30383, 216, 256, "f16", 1, 1, 0),
    (76, 6889, 3980, "f16", 1, 1, 1), (13024, 9665, 21, "f32", 1, 1, 1), (68, 7738, 5521, "f32", 0, 0, 1), (78579, 1866, 21, "bf16", 1, 0, 1),
    (8108, 75, 5183, "bf16", 0, 1, 1), (7204, 73, 6054, "f16", 1, 0, 1), (8179, 76, 5903, "bf16", 1, 0, 0), (101439, 1511, 24, "f16", 1, 1, 1),
    (67, 7965, 7040, "f16", 0, 1, 0), (15443, 17859, 144, "bf16", 1, 1, 0), (9370, 42319, 133, "f16", 1, 1, 0)
]

LOSS = r"""
#include <stdio.h>
#include "paper_2206_08869_amd/csrc/loss_plan.h"
int main() {
    long long rows; int classes, cols, type, backward, live, aligned;
    while (scanf("%lld %d %d %d %d %d %d", &rows, &classes, &cols, &type, &backward, &live, &aligned) == 7) {
        iodf_class_loss a{};
        a.rows = rows, a.classes = classes, a.cols = cols, a.type = type;
        a.u = a.w = (void*)(size_t)(aligned ? 256 : 252), a.u_stride = a.w_stride = aligned ? (cols + 7) / 8 * 8 : cols + 1;
        a.live = live ? (uint8_t*)256 : nullptr, a.du = a.dw = (void*)256;
        const iodf::LossPlan p = iodf::loss_plan(a, backward);
        printf("%d %d %d %d %d %d %d %d %d %d %lld\n", p.few, p.few_rows, p.fine, p.logits.edge, p.logits.slices, p.du.edge, p.du.slices, p.dw.edge, p.dw.slices,
               (int)p.together, p.piece);
    }
}
"""
ORTH = r"""
#include <stdio.h>
#include "paper_2206_08869_amd/csrc/orth_plan.h"
int main() {
    long long count; int rows, cols, type;
    while (scanf("%lld %d %d %d", &count, &rows, &cols, &type) == 4) {
        const iodf::OrthPlan p = iodf::orth_plan(iodf::together(count, rows, cols), rows, cols, type);
        printf("%d %d %d %d %d %d %d %d %d %d\n", (int)p.block, p.groups, p.per, (int)p.tall, (int)p.parts, p.first.edge, p.first.pieces, p.second.edge, p.second.pieces, p.apply_edge);
    }
}
"""


def _run(source, lines):
    with tempfile.TemporaryDirectory() as d:
        with open(os.path.join(d, "plan.cpp"), "w") as f:
            f.write(source)
        exe = os.path.join(d, "plan")
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wno-unused-function", "-I", ROOT, f.name, "-o", exe], check=True)
        out = subprocess.run([exe], input="\n".join(" ".join(str(int(x)) for x in line) for line in lines), capture_output=True, text=True, check=True).stdout
    got = [[int(x) for x in line.split()] for line in out.splitlines()]
    assert len(got) == len(lines)
    return got


def orth_kinds(shapes):
    """Of each (count, rows, cols, type name): the kernels that it takes, as tuples."""
    out = []
    for block, groups, per, tall, parts, e1, p1, e2, p2, apply in _run(ORTH, [(n, r, c, TYPES[t]) for n, r, c, t in shapes]):
        products = 3 if parts else 1
        if block:
            kinds = {("one block", products)}
        elif groups:
            kinds = {("slim", "at once" if groups == 1 else "step by step", "one block each" if per == 1 else "several", "tall" if tall else "wide", products)}
        else:
            way = "tall" if tall else "wide"
            kinds = {("first", e1, "pieces" if p1 else "tiles", way, products), ("second", e2, "pieces" if p2 else "tiles", products), ("apply", apply, way, products)}
        out.append(kinds)
    return out


def loss_kinds(calls):
    """Of each (rows, classes, cols, type name, backward, live, aligned): the kernels that it takes, as tuples."""
    out = []
    for call, (few, few_rows, fine, edge, slices, du, du_slices, dw, dw_slices, both, piece) in zip(calls, _run(LOSS, [(*c[:3], TYPES[c[3]], *c[4:]) for c in calls])):
        name, backward = call[3], call[4]
        if few:
            out.append({("few gradients", few_rows) if backward else ("few", name, few)})
            continue
        how = name + (" in two parts" if fine else "")
        kinds = {("gradient's logits" if backward else "logits", how, edge, "sliced" if slices > 1 else "whole")}
        if backward:
            kinds.add(("gradients", how, du, "together") if both else ("du", how, du))
            if not both:
                kinds.add(("dw", how, dw))
            if du_slices > 1:
                kinds.add(("du joined", how, du))
            if dw_slices > 1:
                kinds.add(("dw joined", how, dw))
            if piece < call[1]:
                kinds.add(("pieces", how))
        out.append(kinds)
    return out
