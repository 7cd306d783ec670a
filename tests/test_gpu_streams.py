"""GPU: the classifier's calls with a stream of their own (`stream=`): what they return belongs
to that stream's memory, and holds what the call on the current stream gives."""

import numpy as np
import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def pid():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2009_04509_amd import binding
    return binding


@pytest.fixture(scope="module")
def calls(pid):
    plane = synth.config1()
    image = torch.from_numpy(plane.image).to(DEV)
    hits = torch.from_numpy(np.ascontiguousarray(plane.hits, dtype=np.int32)).to(DEV)
    hits3 = torch.cat([torch.zeros_like(hits[:, :1]), hits], 1).contiguous()
    patches = pid.pointid_gather(image, hits)
    h = pid.pointid_create(synth.he_normal_weights(), "fp16", 0)
    batcher = pid.Batcher(h, [image])
    torch.cuda.synchronize()

    def found(s):
        at, n = pid.pointid_find_hits(h, [image], 0.5, capacity=4096, stream=s)
        return [n, at]

    yield {
        "classify": lambda s: [pid.pointid_classify(h, image, hits, stream=s)],
        "planes": lambda s: [pid.pointid_classify_planes(h, [image], hits3, stream=s)],
        "planes_noalloc": lambda s: [pid.pointid_classify_planes_noalloc(h, [image], hits3, stream=s)],
        "planes_ds": lambda s: [pid.pointid_classify_planes_ds(h, [image], hits3, 2, stream=s)],
        "requests": lambda s: pid.pointid_classify_requests(h, [image], [(0, hits, None), (-1, hits3, None)], stream=s),
        "patches": lambda s: [pid.pointid_classify_patches(h, patches, stream=s)],
        "gather": lambda s: [pid.pointid_gather(image, hits, "bf16", stream=s)],
        "gather_planes": lambda s: [pid.pointid_gather_planes([image], hits3, stream=s)],
        "downsample": lambda s: [pid.pointid_downsample(image, 3, stream=s)],
        "find_hits": found,
        "batcher": lambda s: [batcher.wait(batcher.submit(0, hits, stream=s))],
    }
    batcher.close()
    h.close()


def pool_of(t):
    """The stream whose memory a tensor has."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's memory")


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", ["classify", "planes", "planes_noalloc", "planes_ds", "requests", "patches", "gather",
                                  "gather_planes", "downsample", "find_hits", "batcher"])
def test_outputs_are_of_the_calls_stream(calls, name, raw):
    call = calls[name]
    want = [t.clone() for t in call(None)]              # and leaves the current stream blocks of the same sizes
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(s.cuda_stream if raw else s)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert pool_of(a) == s.cuda_stream
        if name == "find_hits" and a.dim() == 2:         # only the rows found are written
            n = min(int(got[0]), 4096)
            a, b = a[:n], b[:n]
        assert torch.equal(a, b)
