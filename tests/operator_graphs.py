"""Taskgraphs of a few vertices built by hand, for tests of single operators: inputs from arrays, one run, results as float64."""
import numpy as np
import torch

from paper_2405_16283_amd import binding as B
from workloads import bf16_bits_to_f32, to_bf16_bits

CODE = {"f32": B.TN_F32, "bf16": B.TN_BF16, "i32": B.TN_I32}


def rounded(a, dtype):
    """`a` as stored in dtype, in float64."""
    a = np.ascontiguousarray(a, dtype=np.float32)
    return (a if dtype == "f32" else bf16_bits_to_f32(to_bf16_bits(a).reshape(a.shape))).astype(np.float64)


class Graph:
    def __init__(self, dtype="f32"):
        self.dtype = dtype
        self.tg = B.tn_taskgraph_create()
        self.host = {}
        self.keep = None

    def inp(self, a, dtype=None):
        dtype = dtype or self.dtype
        a = np.atleast_2d(a)
        if dtype == "i32":
            t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32))
        elif dtype == "f32":
            t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
        else:
            t = torch.from_numpy(to_bf16_bits(np.ascontiguousarray(a, dtype=np.float32)).reshape(a.shape).view(np.int16))
        v = B.tn_taskgraph_add_input(self.tg, CODE[dtype], a.shape[0], a.shape[1], B.TN_HOST)
        self.host[v] = t
        return v

    def grid(self, a, row_step, col_step, dtype=None, transposed=False):
        """Input vertices of the array's tiles, by rows of tiles."""
        a = np.atleast_2d(a)
        tiles = [a[r:r + row_step, c:c + col_step] for r in range(0, a.shape[0], row_step) for c in range(0, a.shape[1], col_step)]
        return [self.inp(x.T if transposed else x, dtype) for x in tiles]

    def op(self, kind, ins, rows, cols, dtype=None, **params):
        return B.tn_taskgraph_add_op(self.tg, kind, B.tn_op_params(**params), ins, CODE[dtype or self.dtype], rows, cols)

    def run(self, outs, seed=1, cap=None, static=False):
        """The vertices' tensors, float64, each guarded: bytes behind every result are looked at."""
        shapes = []
        for v in outs:
            B.tn_taskgraph_mark_output(self.tg, v)
            x = B.tn_taskgraph_vertex(self.tg, v).desc
            shapes.append((x.rows, x.cols, x.dtype))
        n = B.tn_taskgraph_num_vertices(self.tg)
        cap = cap or 256 << 20
        mg = B.tn_compile(self.tg, None, cap, None)
        dev = torch.empty(cap, dtype=torch.uint8, device="cuda:0")
        streams = [torch.cuda.Stream() for _ in range(4)]
        host = {v: t.pin_memory() for v, t in self.host.items()}
        size = lambda s: s[0] * s[1] * (2 if s[2] == B.TN_BF16 else 4)  # noqa: E731
        bufs = [torch.full((size(s) + 256,), 0x5A, dtype=torch.uint8).pin_memory() for s in shapes]
        torch.cuda.synchronize()
        ex = B.tn_executor_create(mg, dev.data_ptr(), cap, 0, 0, [streams[0].cuda_stream, streams[3].cuda_stream], streams[1].cuda_stream,
                                  streams[2].cuda_stream)
        try:
            ptrs = [host[v].data_ptr() if v in host else 0 for v in range(n)]
            call = B.tn_execute_static if static else B.tn_execute
            call(ex, ptrs, [b.data_ptr() for b in bufs], B.tn_exec_opts(policy=B.TN_POLICY_RANDOM, order_seed=seed))
        finally:
            B.tn_executor_destroy(ex)
            B.tn_memgraph_destroy(mg)
            B.tn_taskgraph_destroy(self.tg)
        out = []
        for b, s in zip(bufs, shapes):
            assert bool((b[size(s):] == 0x5A).all())
            a = b[:size(s)].numpy()
            a = a.view(np.float32).astype(np.float64) if s[2] == B.TN_F32 else bf16_bits_to_f32(a.view(np.uint16)).astype(np.float64)
            out.append(a.reshape(s[0], s[1]))
        return out
