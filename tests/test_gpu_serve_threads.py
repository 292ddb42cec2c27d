"""Several host threads on ONE stream: calls of several launches that share the stream's workspace, of different sizes, give
what each gives alone."""
import threading

import numpy as np
import pytest

import paper_2607_04031_amd as tl
from tests import test_gpu_attn as attn
from tests import test_gpu_verify as ver
from tests._gpu import banner

pytestmark = pytest.mark.gpu
_lib = attn._lib
CALLS = 100


def test_attention_verification_and_products_on_one_stream():
    import torch
    banner("tl_attn, tl_verify and split-K tl_gemm from four host threads on one stream")
    i32, f32 = torch.int32, torch.float32
    a = attn.Case(90, [5000, 1200], [1, 3], 8, 1, 128, 1, 64)
    a_args = [a.q_dev(), a.cache.device(), attn._int(a.table), attn._int(a.lens), attn._int(a.offsets), 3, 5000, a.scale]
    work = {"attention": lambda out: tl.attention(*a_args, out=out, stream=side),
            "another attention": lambda out: tl.attention(*a_args[:5], 60, 100000, a.scale, out=out, stream=side)}
    outs = {n: torch.empty((4, 8, 128), dtype=torch.bfloat16, device="cuda") for n in work}
    c, _, _ = ver._case(91, [24, 7], 40000, 3, "f32", False)
    dev = ver._dev
    v_args = [dev(c["logits"], f32), dev(c["offsets"], i32), dev(c["parents"], i32), dev(c["tokens"], i32), dev(c["temperature"], f32),
              dev(c["uniform"], f32), dev(c["noise"], f32), c["max_nodes"]]
    draft = dev(c["draft"], f32)
    work["verification"] = lambda out: tl.verify(*v_args, draft=draft, out=out, stream=side)
    outs["verification"] = tuple(torch.empty(n, dtype=i32, device="cuda") for n in ((2, c["max_nodes"]), 2, 2))
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(8, 8192, generator=g, device="cuda").to(torch.bfloat16)
    w = tl.repack(torch.randn(2048, 8192, generator=g, device="cuda").to(torch.bfloat16))
    work["product"] = lambda out: tl.gemm(x, w, 2048, tl.layout(split_k=4), out=out, stream=side)
    outs["product"] = torch.empty((8, 2048), dtype=f32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def flat(name):
        side.synchronize()
        return [t.cpu().clone() for t in (outs[name] if isinstance(outs[name], tuple) else (outs[name],))]

    want = {}
    for name, call in work.items():
        call(outs[name])
        want[name] = flat(name)
    assert int(want["verification"][1].max()) > 1 and all(t.any() for w in want.values() for t in w)
    errors = []

    def run(name, start):
        try:
            start.wait()
            for _ in range(CALLS):
                work[name](outs[name])
        except Exception as e:              # reported on the main thread
            errors.append((name, e))

    for turn in range(3):
        for x_ in outs.values():
            for t in x_ if isinstance(x_, tuple) else (x_,):
                t.zero_()
        torch.cuda.synchronize()
        start = threading.Barrier(len(work))
        threads = [threading.Thread(target=run, args=(name, start)) for name in work]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not errors, errors
        for name in work:
            for got, ref in zip(flat(name), want[name]):
                np.testing.assert_array_equal(got.float().numpy(), ref.float().numpy(), err_msg=name)
