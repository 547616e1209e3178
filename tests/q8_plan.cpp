// q8_plan.cpp -- the host side of the operators on 8-bit rows without a GPU: the source itself, with every launch
// printed instead of made.  One query per line of standard input, one line of output per query:
//
//   plan N nnz F W mode n_rows      ->  the product's plan, as "name value" pairs
//   bytes N nnz F W mode n_rows     ->  es_spmm_q8_workspace_bytes
//   write type n F rows N           ->  status, then per launch "blocks threads rows first" (first: of the table)
//   read type n F rows N            ->  the same
//   spmm N nnz F W mode n_rows ws   ->  status, then per launch "blocks threads"; ws: the asked workspace is given
//   vals N nnz F W mode             ->  the same
//   grad N F H ws                   ->  the same
//
// `rows` says whether ids are given.  The addresses are never read.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <iostream>
#include <sstream>
#include <string>

namespace {
template <class... A> void record(dim3 grid, dim3 block, const A&... args);
}

#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) record(grid, block, __VA_ARGS__)
#define hipGetLastError() hipSuccess
#include "es_q8.hip"

namespace {

std::ostringstream launches;
char* const kTable = reinterpret_cast<char*>(uintptr_t(1) << 40);          // where the codes begin

void detail(const Q8Write& a) { launches << ' ' << a.n << ' ' << ((char*)a.codes - kTable) / a.ldq; }
void detail(const Q8Read& a) { launches << ' ' << a.n << ' ' << ((char*)a.codes - kTable) / a.ldq; }
template <class... A> void detail(const A&...) {}

template <class... A> void record(dim3 grid, dim3 block, const A&... args)
{
    launches << ' ' << (uint64_t)grid.x << ' ' << (uint64_t)block.x;
    detail(args...);
}

template <class T> T* fake(uintptr_t at) { return reinterpret_cast<T*>(at); }

}  // namespace

int main()
{
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        std::string what;
        in >> what;
        launches.str("");
        int64_t v[8] = {};
        for (int i = 0; i < 8 && in >> v[i]; ++i) {}
        int8_t* codes = reinterpret_cast<int8_t*>(kTable);
        float* scale = fake<float>(uintptr_t(1) << 41);
        int32_t* graph = fake<int32_t>(uintptr_t(1) << 42);
        float* dense = fake<float>(uintptr_t(1) << 43);
        void* ws = fake<void>(uintptr_t(1) << 44);
        if (what == "plan") {
            const Q8Plan p = plan_q8(v[0], v[1], (int32_t)v[2], (int32_t)v[3], (int32_t)v[4], v[5]);
            std::cout << "few " << p.few << " splits " << p.splits << " piece " << p.piece << " pieces " << p.pieces << " long_k "
                      << p.long_k << " long_blocks " << p.long_blocks << " grid_x " << p.grid_x << " team " << p.team << " G " << p.G
                      << " wave_rows " << p.wave_rows << " nblocks " << p.nblocks << "\n";
        } else if (what == "bytes") {
            std::cout << es_spmm_q8_workspace_bytes(v[0], v[1], (int32_t)v[2], (int32_t)v[3], (int32_t)v[4], v[5]) << "\n";
        } else {
            int rc = 1;
            if (what == "write")
                rc = es_q8_write(dense, (int32_t)v[0], v[1], (int32_t)v[2], (int32_t)v[2], v[3] ? graph : nullptr, v[4], codes,
                                 es_q8_row_bytes((int32_t)v[2]), scale, nullptr);
            else if (what == "read")
                rc = es_q8_read(codes, es_q8_row_bytes((int32_t)v[2]), scale, v[4], (int32_t)v[2], v[3] ? graph : nullptr, v[1], dense,
                                (int32_t)v[0], (int32_t)v[2], nullptr);
            else if (what == "spmm")
                rc = es_spmm_q8(graph, graph, nullptr, codes, es_q8_row_bytes((int32_t)v[2]), scale, dense, v[0], v[1], (int32_t)v[2],
                                (int32_t)v[2], (int32_t)v[3], (int32_t)v[4], 0, 0, graph, v[5], v[6] ? ws : nullptr,
                                v[6] ? es_spmm_q8_workspace_bytes(v[0], v[1], (int32_t)v[2], (int32_t)v[3], (int32_t)v[4], v[5]) : 0,
                                nullptr);
            else if (what == "vals")
                rc = es_spmm_q8_backward_vals(graph, graph, dense, (int32_t)v[2], codes, es_q8_row_bytes((int32_t)v[2]), scale, dense,
                                              v[0], v[1], (int32_t)v[2], (int32_t)v[3], (int32_t)v[4], 0, 0, nullptr);
            else if (what == "grad")
                rc = es_q8_weight_grad(codes, es_q8_row_bytes((int32_t)v[1]), scale, dense, (int32_t)v[2], dense, (int32_t)v[2], v[0],
                                       (int32_t)v[1], (int32_t)v[2], v[3] ? ws : nullptr,
                                       v[3] ? es_q8_weight_grad_workspace_bytes(v[0], (int32_t)v[1], (int32_t)v[2]) : 0, nullptr);
            std::cout << rc << launches.str() << "\n";
        }
    }
    return 0;
}
