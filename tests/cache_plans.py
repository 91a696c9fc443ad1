"""How the library splits a cache call over CTAs, worked out again from the sizes: tests name the split they
mean to reach and assert that they reach it; and the launches that a call really makes."""
import ctypes as C


def stages(dim):
    return 6 if dim == 256 else 3


def attend_split(lens, heads, dim, max_len, scored, masked, sms=148):
    """{"cluster": CTAs per row, "each": tiles of a CTA} or {"cluster": 0, "each", "with_rows", "parts": per non-empty row, if shares
    end with rows}.  (At 256 channels: as long as the rows' clusters fit the GPU at once.)"""
    up = lambda a, b: -(-a // b)
    tile = 8192 // dim
    rows, row_tiles, limit = len(lens) * heads, up(max_len, tile), sms * (1 if dim == 256 else 2)
    most, size = 8 if dim == 256 else 16, 1
    while size < most and size < row_tiles and rows * size * 2 <= sms:
        size *= 2
    many = rows * 2 > limit
    if row_tiles <= size * (16 if many else 6) and (many or not scored):
        return {"cluster": size, "each": up(up(max(lens), tile), size)}
    grid = min(limit, rows * row_tiles)
    tiles = [up(n, tile) for n in lens]
    each = max(1, up(sum(tiles) * heads, grid))
    if each >= 6 and not masked:
        for k in range(4):
            e = each + k * (each // 6) // 3
            if sum(up(t, e) for t in tiles) * heads <= grid:
                return {"cluster": 0, "each": e, "with_rows": True, "parts": sorted({up(t, e) for t in tiles if t})}
    return {"cluster": 0, "each": each, "with_rows": False}


def select_split(rows, max_len, sms=148, fit={2: 74, 4: 33, 8: 15}):
    """(CTAs per row, keys per thread that the kernel is built for; 0: keys read again for every step).  `fit`: clusters with an SM to each CTA
    that the GPU holds at once; test_gpu_cache_splits.py asks for no split that a few more or less would change."""
    size = 1
    while size < 8 and (size * 1024 * 33 < max_len or (rows * size * 2 <= sms and rows <= fit[size * 2] and size * 1024 * 3 < max_len)):
        size *= 2
    per = -(-max_len // (size * 1024))
    return size, next((k for k in (3, 9, 17, 25, 33) if per <= k), 0)


class _KernelNode(C.Structure):
    _fields_ = [("func", C.c_void_p), ("grid", C.c_uint * 3), ("block", C.c_uint * 3), ("smem", C.c_uint), ("params", C.c_void_p),
                ("extra", C.c_void_p), ("kern", C.c_void_p), ("ctx", C.c_void_p)]


class _Attribute(C.Structure):
    _fields_ = [("id", C.c_int), ("pad", C.c_char * 4), ("cluster", C.c_uint * 3), ("rest", C.c_char * 52)]


class _LaunchConfig(C.Structure):
    _fields_ = [("grid", C.c_uint * 3), ("block", C.c_uint * 3), ("smem", C.c_uint), ("stream", C.c_void_p), ("attrs", C.POINTER(_Attribute)),
                ("count", C.c_uint)]


def launches(call):
    """The kernels that `call` launches (captured in a graph, not run), in order: nodes with grid, block and smem."""
    import torch
    cu = C.CDLL("libcuda.so.1")
    call()                                                  # buffers and attributes that a first call makes
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw, n = C.c_void_p(graph.raw_cuda_graph()), C.c_size_t()
    assert cu.cuGraphGetNodes(raw, None, C.byref(n)) == 0
    nodes = (C.c_void_p * n.value)()
    assert cu.cuGraphGetNodes(raw, nodes, C.byref(n)) == 0
    out = []
    for node in nodes:
        p = _KernelNode()
        assert cu.cuGraphKernelNodeGetParams_v2(C.c_void_p(node), C.byref(p)) == 0
        out.append(p)
    return out


def resident_clusters(node, size):
    """How many clusters of `size` of a launch's blocks the GPU holds at once."""
    cu = C.CDLL("libcuda.so.1")
    func, n = C.c_void_p(node.func), C.c_int()
    if not func:
        assert cu.cuKernelGetFunction(C.byref(func), C.c_void_p(node.kern)) == 0
    cluster = _Attribute()
    cluster.id, cluster.cluster[:] = 4, (size, 1, 1)        # CU_LAUNCH_ATTRIBUTE_CLUSTER_DIMENSION
    config = _LaunchConfig(node.grid, node.block, node.smem, None, C.pointer(cluster), 1)
    assert cu.cuOccupancyMaxActiveClusters(C.byref(n), func, C.byref(config)) == 0
    return n.value
