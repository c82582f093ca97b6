"""Which lists a step refuses for memory that two of its buffers share (csrc/param_ranges.h), without a GPU: every pair of buffers of one tensor and of two, against a comparison of
all pairs in lists of any order."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <random>

#include "param_ranges.h"

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); std::exit(1); } } while (0)

static void *at(uint64_t p) { return reinterpret_cast<void *>(p); }

// Tensor number i of n elements with buffers of its own, 1 MiB apart: fp32 weight, bf16 gradient, f16 copy, 8-bit moments.
static mqg_param tensor(uint64_t i, int64_t n) {
    mqg_param p = {};
    const uint64_t base = (uint64_t(7) << 40) + i * (16 << 20);
    p.numel = n;
    p.weight = at(base);
    p.grad = at(base + (1 << 20));
    p.copy = at(base + (2 << 20));
    p.m = at(base + (3 << 20));
    p.v = at(base + (4 << 20));
    p.m_scale = static_cast<float *>(at(base + (5 << 20)));
    p.v_scale = static_cast<float *>(at(base + (6 << 20)));
    p.weight_type = MQG_F32;
    p.grad_type = MQG_BF16;
    p.copy_type = MQG_F16;
    p.state_type = MQG_STATE_E4M3;
    return p;
}
constexpr int kBuffers = 7, kGrad = 1;
static uint64_t get(const mqg_param &p, int b) {
    const void *all[] = {p.weight, p.grad, p.copy, p.m, p.v, p.m_scale, p.v_scale};
    return reinterpret_cast<uint64_t>(all[b]);
}
static void set(mqg_param &p, int b, uint64_t v) {
    if (b == 0) p.weight = at(v);
    if (b == 1) p.grad = at(v);
    if (b == 2) p.copy = at(v);
    if (b == 3) p.m = at(v);
    if (b == 4) p.v = at(v);
    if (b == 5) p.m_scale = static_cast<float *>(at(v));
    if (b == 6) p.v_scale = static_cast<float *>(at(v));
}
static uint64_t size_of(const mqg_param &p, int b) {
    const uint64_t n = static_cast<uint64_t>(p.numel), scales = (n + 127) / 128 * 4;
    const bool eight = p.state_type == MQG_STATE_E4M3;
    const uint64_t of[] = {n * (p.weight_type == MQG_F32 ? 4 : 2), n * (p.grad_type == MQG_F32 ? 4 : 2), p.copy ? n * (p.copy_type == MQG_F32 ? 4 : 2) : 0, n * (eight ? 1 : 4),
                           n * (eight ? 1 : 4), eight ? scales : 0, eight ? scales : 0};
    return of[b];
}
static bool shares(const std::vector<mqg_param> &l) { return mqg::step_shares_memory(l.data(), static_cast<int32_t>(l.size()), {}); }

int main() {
    CHECK(!shares({}));
    CHECK(!shares({tensor(0, 300), tensor(1, 1), tensor(2, 100000)}));
    for (int64_t n : {1, 128, 300}) {
        // one buffer where another begins, and on its last byte, of the same tensor (k = 0) and of two; the first byte behind it is free
        for (int k = 0; k < 2; ++k)
            for (int a = 0; a < kBuffers; ++a)
                for (int b = 0; b < kBuffers; ++b) {
                    if (k == 0 && a == b) continue;
                    for (int order = 0; order < 2; ++order) {
                        std::vector<mqg_param> l = {tensor(0, n), tensor(1, n)};
                        mqg_param &to = l[order ? 1 - k : k], &from = l[order ? 1 : 0];
                        const uint64_t begin = get(from, b), last = begin + size_of(from, b) - 1;
                        const bool both_read = a == kGrad && b == kGrad;
                        set(to, a, begin);
                        CHECK(shares(l) == !both_read);
                        set(to, a, last);
                        CHECK(shares(l) == !both_read);
                        set(to, a, last + 1);
                        CHECK(!shares(l));
                    }
                }
    }
    // what is not there, and what is not stepped, shares nothing
    std::vector<mqg_param> l = {tensor(0, 300), tensor(0, 300)};
    CHECK(shares(l));
    l[1].grad = nullptr;
    CHECK(!shares(l));
    l[1] = tensor(0, 0);
    CHECK(!shares(l));
    l[1] = tensor(1, 300);
    l[1].copy = nullptr;
    l[0].copy = nullptr;
    l[0].state_type = l[1].state_type = MQG_STATE_F32;
    l[1].m_scale = l[0].m_scale = l[0].v_scale;
    CHECK(!shares(l));
    l[0].m = at(get(l[0], 4) - 4 * 300);
    CHECK(!shares(l));
    l[0].m = at(get(l[0], 4) - 4 * 300 + 1);
    CHECK(shares(l));
    // numbers that are read on the device
    l = {tensor(0, 300)};
    const void *in = at(get(l[0], 0) + 40), *in_grad = at(get(l[0], kGrad) + 40), *out = at(64);
    CHECK(!mqg::step_shares_memory(l.data(), 1, {{nullptr, 8}, {out, 4}, {out, 4}, {in_grad, 4}}));
    CHECK(mqg::step_shares_memory(l.data(), 1, {{out, 8}, {in, 4}}));
    CHECK(mqg::step_shares_memory(l.data(), 1, {{at(get(l[0], 5) + 8), 4}, {out, 4}}));

    std::mt19937_64 rng(1);
    int found = 0;
    for (int round = 0; round < 4000; ++round) {
        l.clear();
        const int count = 1 + static_cast<int>(rng() % 6);
        for (int i = 0; i < count; ++i) {
            mqg_param p = tensor(0, static_cast<int64_t>(rng() % 40));
            for (int b = 0; b < kBuffers; ++b) set(p, b, 64 + rng() % 4000 * 4);
            p.weight_type = static_cast<int32_t>(rng() % 3);
            p.grad_type = static_cast<int32_t>(rng() % 3);
            p.state_type = static_cast<int32_t>(rng() % 2);
            if (rng() % 2) p.copy = nullptr;
            if (rng() % 8 == 0) p.grad = nullptr;
            l.push_back(p);
        }
        bool want = false;
        for (int i = 0; i < count; ++i)
            for (int j = 0; j <= i; ++j)
                for (int a = 0; a < kBuffers; ++a)
                    for (int b = 0; b < kBuffers; ++b) {
                        if ((i == j && a <= b) || (a == kGrad && b == kGrad) || !l[i].grad || !l[j].grad) continue;
                        const uint64_t x = get(l[i], a), y = get(l[j], b), nx = size_of(l[i], a), ny = size_of(l[j], b);
                        want |= nx && ny && x < y + ny && y < x + nx;
                    }
        CHECK(shares(l) == want);
        found += want;
    }
    CHECK(found > 400 && found < 3600);
    std::puts("ok");
}
"""


def test_every_pair_of_buffers(tmp_path):
    src, exe = tmp_path / "ranges.cpp", tmp_path / "ranges"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2601_04707_amd", "csrc"), "-I", os.path.join(ROOT, "include"),
                           "-o", str(exe), str(src)])
    done = subprocess.run([str(exe)], text=True, capture_output=True)
    assert done.stdout.strip() == "ok" and done.returncode == 0, done.stdout
