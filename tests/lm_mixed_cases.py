"""Graphs in which the language-model operators meet each other and the older ones in orders other than a layer's own."""
from paper_1707_08265_b200 import workloads as wl

SUM_READERS = ("scales of rows", "scales of tiles", "given scales", "norm over tensors", "clipped", "scan of it", "scan gated by it", "gain of another norm")


def sum_read_before_its_norm(reader, dtype, rows=70, cols=264):
    """h = Add(x, r), fetched; an operator that reads h; then RMSNorm(h).  Returns (graph, inputs, outputs: h, the reader's, y)."""
    g = wl.GraphDesc()
    shape = [cols] if reader == "gain of another norm" else [rows, cols]
    blocks = -(-cols // 128)
    x, r, w = g.tensor("x", shape, dtype), g.tensor("r", shape, dtype), g.tensor("w", [cols])
    inputs = [x, r, w]
    h = g.op("Add", [x, r], "h", shape, dtype)
    if reader == "scales of rows":
        s = g.op("BlockScale", [h], "s", [rows, blocks], attrs=[1])
        read = [s, g.op("Quantize", [h, s], "q", shape, "f8e4m3")]
    elif reader == "scales of tiles":
        read = [g.op("BlockScale", [h], "s", [-(-rows // 128), blocks], attrs=[128])]
    elif reader == "given scales":
        s = g.tensor("s", [rows, blocks])
        inputs.append(s)
        read = [g.op("Quantize", [h, s], "q", shape, "f8e4m3")]
    elif reader == "norm over tensors":
        read = [g.op("GlobalNorm", [x, h], "n", [])]
    elif reader == "clipped":
        n = g.op("GlobalNorm", [h], "n", [])
        read = [n, g.op("ClipByNorm", [h, n], "c", shape, dtype, attrs=[0.5])]
    elif reader == "gain of another norm":
        z = g.tensor("z", [3, cols])
        inputs.append(z)
        read = [g.op("RMSNorm", [z, h], "yz", [3, cols])]
    else:
        z = g.tensor("z", shape, dtype)
        inputs.append(z)
        read = [g.op("GatedScan", [z, h] if reader == "scan of it" else [h, z], "states", shape, dtype)]
    y = g.op("RMSNorm", [h, w], "y", shape, dtype)
    return g, inputs, [h] + read + [y]
